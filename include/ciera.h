/*
 * ciera.h -- C ABI of the B200 (sm_100a) exponent-reuse codec.
 *
 * The library implements the data-parallel hot path of CIERA's "Exponent Reuse based
 * Compression" (paper Section 3.1, Algorithm 1) and the gain rule of "Benefit-driven
 * Selective Compression" (Section 3.2):
 *
 *   sender    split every weight into exponent and sign-plus-mantissa, compare the exponents
 *             with a cached copy block by block, emit (bitmap, sign-plus-mantissa of all
 *             values, exponents of changed blocks), refresh the cache for changed blocks;
 *   receiver  patch its exponent cache with the changed blocks, merge cache and
 *             sign-plus-mantissa back into bit-identical weights.
 *
 * Conventions
 *   - Every function returns a ciera_status (0 = CIERA_OK, negative = error).  Nothing throws,
 *     nothing is printed, and no codec state lives in the library: caches, messages and scratch
 *     are the caller's buffers.  What the library does keep per process: the launch counter, the
 *     thread's last CUDA error, per device the grid sizes and attributes it has worked out for its kernels, and up to
 *     eight pairs of copy streams with their events, made by ciera_roundtrip_host when it first needs
 *     them (all but one pair are given up when the last plan is destroyed).
 *   - "dev" pointers are CUDA device pointers, "host" pointers are ordinary host pointers.
 *     The library never allocates device memory: the caller owns every device buffer and
 *     passes scratch space explicitly.  The only host allocations are the plan object and the
 *     records of those copy streams.  (One
 *     exception, stated where it is declared: ciera_encode_noalloc works in a fixed device array
 *     that is part of the library image, for callers that cannot supply scratch.)
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Device work is
 *     enqueued on it and the call returns without waiting, unless stated otherwise.
 *     The sender, transport, receiver and entropy calls read every size they need on the device
 *     and leave their scratch as they found it, so a step may be captured in a CUDA graph and
 *     replayed; call each entry point once outside a capture first (its first call on a device
 *     queries occupancy and sets kernel attributes).  The host-side launch counter does not see
 *     replays.
 *   - Errors found on the device (a wait that ran out, a message whose length contradicts its
 *     bitmap) are written to the caller's `status_dev` word: 0 = none, otherwise the first
 *     ciera_status that was raised.  The word is only ever written on error; clear it yourself.
 *   - A *unit* is one shard of one tensor: N consecutive values.  Units are independent; one call
 *     processes a whole table of them ("batched launch over simulated shards").
 *
 * Wire format of one unit's message (b bits per value, m = b - 8 sign-plus-mantissa bits,
 * block size B, nb = ceil(N/B) blocks; Section 3.2 for the sizes, Algorithm 1 for the order
 * bitmap, mant, payload):
 *
 *   [ bitmap : ceil(nb/8) bytes, block k -> byte k>>3 bit k&7, unused high bits 0 ]
 *   [ zero pad to a multiple of 16 ]
 *   [ sm     : N*m/8 bytes; bf16: byte j = sign<<7 | mantissa(7);
 *              fp32: bytes 3j..3j+2 = (sign<<23 | mantissa(23)) little-endian ]
 *   [ zero pad to a multiple of 16 ]
 *   [ payload: for every changed block in ascending k, its exponent bytes (B of them, fewer
 *              for a short last block) ]
 *
 * No header travels: the payload length follows from the bitmap.  The paper's byte count
 * S_{s+m} + S_bm + (changed exponent bytes) is ciera_message_bytes(); the length that has to
 * be moved (it includes the two pads, at most 30 bytes) is what ciera_encode reports.
 * Bytes of a slot past the reported length are unspecified.
 */
#ifndef CIERA_H
#define CIERA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define CIERA_API __attribute__((visibility("default")))
#else
#define CIERA_API
#endif

typedef enum ciera_status {
    CIERA_OK = 0,
    CIERA_ERR_INVALID_ARG = -1, /* null pointer, zero block, bad enum, inconsistent sizes      */
    CIERA_ERR_UNSUPPORTED = -2, /* block size outside the supported set                         */
    CIERA_ERR_MISALIGNED = -3,  /* an offset or base pointer is not a multiple of 16 bytes      */
    CIERA_ERR_CAPACITY = -4,    /* a message slot, plan image or scratch buffer is too small    */
    CIERA_ERR_CUDA = -5,        /* a CUDA runtime call failed (see ciera_last_cuda_error)       */
    CIERA_ERR_TIMEOUT = -6,     /* device: a bounded wait on another tile ran out               */
    CIERA_ERR_CORRUPT = -7,     /* device: message length disagrees with its bitmap             */
    CIERA_ERR_NOT_BOUND = -8,   /* the plan has no device image yet (ciera_plan_bind)           */
    CIERA_ERR_TOO_LARGE = -9    /* more tiles than the built-in scratch of ciera_encode_noalloc */
} ciera_status;

typedef enum ciera_dtype {
    CIERA_BF16 = 0, /* b = 16: 1 sign, 8 exponent, 7 mantissa bits  -> m = 8  */
    CIERA_FP32 = 1, /* b = 32: 1 sign, 8 exponent, 23 mantissa bits -> m = 24 */
    CIERA_FP16 = 2  /* b = 16: 1 sign, 5 exponent, 10 mantissa bits -> m = 11 (IEEE binary16).  On the
                       wire its exponents take 5 bits and its sign-plus-mantissa 11 bits each, packed
                       without gaps (value j of a section at bits [j*w, (j+1)*w), bit i of a section =
                       byte i >> 3, bit i & 7); every changed block of the payload starts on a byte
                       boundary (a block of 1, 2, 4, 8, 16 ... values takes 1, 2, 3, 5, 10 ... bytes);
                       the caches still hold one byte per value.  Every block size; the hashed
                       sender takes it too (blocks of 16 values and more, as for the other
                       precisions), and so does the entropy stage, which codes the 5-bit exponents
                       as symbols of their own (it undoes the packing first; 32 table entries
                       travel instead of 256). */
} ciera_dtype;

/* One unit = one shard of one tensor.  All offsets are in BYTES from the base pointer of the
 * respective buffer and must be multiples of 16.  Nothing behind the furthest unit's last value (byte) of a buffer
 * is read or written; between units the rest of a unit's last 16 bytes may be read, and is never used or written. */
typedef struct ciera_unit {
    uint64_t n_values;     /* N; may be 0, may be smaller than the block size                   */
    uint64_t weights_off;  /* into the weights buffer (encode: input, decode: output)           */
    uint64_t cache_off;    /* into the exponent cache (1 byte per value)                        */
    uint64_t msg_off;      /* into the message buffer: start of this unit's slot                */
    uint64_t msg_capacity; /* size of the slot, >= ciera_message_capacity(N, dtype, block)      */
} ciera_unit;

/* ---- sizes (host, pure functions; Section 3.2) ------------------------------------------- */

/* Smallest and largest supported block size B (a power of two in this range).  B = 1 is change
 * detection per value: the bitmap has one bit per value and the payload holds exactly the exponents
 * that changed (Section 2.3: a block stays reusable with probability (1-c)^B, so finer blocks are
 * reused more often, at the price of a longer bitmap). */
#define CIERA_MIN_BLOCK 1u
#define CIERA_MAX_BLOCK 4096u

/* Slot size that always suffices: every block changed (payload = N exponent bytes). */
CIERA_API size_t ciera_message_capacity(uint64_t n_values, int dtype, uint32_t block);
/* Offset of the sign-plus-mantissa section / of the payload section inside a slot. */
CIERA_API size_t ciera_sm_offset(uint64_t n_values, uint32_t block);
CIERA_API size_t ciera_payload_offset(uint64_t n_values, int dtype, uint32_t block);
/* The paper's transmitted bytes S_{s+m} + S_bm + payload_bytes (no pads). */
CIERA_API size_t ciera_message_bytes(uint64_t n_values, int dtype, uint32_t block, uint64_t payload_bytes);

/* ---- plan: the tile table of a unit table -------------------------------------------------- */

/* A plan splits every unit into tiles of ciera_plan_tile_values() consecutive values (one tile
 * is the work of one thread block) and holds the device-side table that the kernels read.  It
 * is immutable after ciera_plan_bind and may be shared by any number of calls and streams. */
typedef struct ciera_plan ciera_plan;

/* Host only.  Validates the units (alignment, capacity, block size) and builds the table.
 * `units_host` is copied.  Destroy with ciera_plan_destroy. */
CIERA_API int ciera_plan_create(const ciera_unit* units_host, uint32_t n_units, int dtype, uint32_t block,
                      ciera_plan** plan_out);
CIERA_API void ciera_plan_destroy(ciera_plan* plan);

CIERA_API uint32_t ciera_plan_n_units(const ciera_plan* plan);
CIERA_API uint32_t ciera_plan_n_tiles(const ciera_plan* plan);
CIERA_API uint32_t ciera_plan_tile_values(const ciera_plan* plan);
CIERA_API uint64_t ciera_plan_total_values(const ciera_plan* plan);
/* Bytes of device memory the table needs (>= 16), and the host image that has to be there. */
CIERA_API size_t ciera_plan_device_bytes(const ciera_plan* plan);
CIERA_API const void* ciera_plan_host_image(const ciera_plan* plan);
/* Bytes of scratch ("workspace") that ciera_encode, ciera_transport and ciera_decode work in: 12 bytes per
 * tile (a look-back status word for the sender, a count for the receiver) and a few counters. */
CIERA_API size_t ciera_plan_workspace_bytes(const ciera_plan* plan);
/* Zero-fills a workspace of ciera_plan_workspace_bytes(plan) bytes (16-byte aligned) on `stream`.  Every
 * call that takes a workspace (ciera_encode, ciera_encode_hashed, ciera_transport, ciera_decode,
 * ciera_roundtrip_host) expects its counters in it all zero when it starts and leaves them all zero when it
 * has finished, so that no launch is spent on clearing them before every call: initialise a workspace once
 * after allocating it, and again after a call whose device status word came back with an error (a kernel
 * that gave up leaves the workspace in an unspecified state).  A plain cudaMemset of the whole workspace
 * does the same. */
CIERA_API int ciera_workspace_init(const ciera_plan* plan, void* workspace_dev, void* stream);

/* Copies the table into caller-owned device memory `plan_dev` (>= ciera_plan_device_bytes,
 * 16-byte aligned) on `stream`, waits for the copy, and remembers the pointer.  The memory must
 * stay valid and unmodified for as long as the plan is used. */
CIERA_API int ciera_plan_bind(ciera_plan* plan, void* plan_dev, size_t plan_dev_bytes, void* stream);

/* ---- caches (Algorithm 1: persistent sender / receiver state) ------------------------------ */

/* cache := exponents of `weights_dev`, or all zero if weights_dev == NULL.  The paper switches
 * its method on once warm-up is over and does not say what the caches hold at that moment;
 * initialising both sides from the same weights (as if they had been sent uncompressed), or
 * both to zero, keeps them in agreement. */
CIERA_API int ciera_cache_init(const ciera_plan* plan, void* cache_dev, const void* weights_dev, void* stream);
/* cache := exponents of `weights_dev`, unconditionally (e.g. after a checkpoint restore). */
CIERA_API int ciera_cache_update(const ciera_plan* plan, void* cache_dev, const void* weights_dev, void* stream);

/* ---- sender: Algorithm 1, sender part; Section 3.1 ----------------------------------------- */

/*
 * For every unit: split, block-wise change detection against `sender_cache_dev`, write the
 * message into the unit's slot of `messages_dev`, refresh the cache for changed blocks.
 *   weights_dev         in   values of the plan's dtype at units[].weights_off
 *   sender_cache_dev    i/o  1 byte per value at units[].cache_off
 *   messages_dev        out  slots at units[].msg_off
 *   wire_bytes_dev      out  [n_units] bytes that have to travel (payload offset + payload bytes;
 *                            0 for an empty unit)
 *   changed_blocks_dev  out  [n_units] number of set bitmap bits
 *   workspace_dev       i/o  scratch of ciera_plan_workspace_bytes(), 16-byte aligned (look-back status
 *                            words, the counter that runs of tiles are handed out from); all zero on
 *                            entry -- see ciera_workspace_init -- and handed back all zero; must not
 *                            be shared by calls that can overlap on the GPU
 *   status_dev          i/o  device error word (may be NULL)
 * One kernel launch for the whole table, nothing else (a table that holds empty units: two small
 * clearing operations in front of it, which write those units' zero lengths and counts).
 */
CIERA_API int ciera_encode(const ciera_plan* plan, const void* weights_dev, void* sender_cache_dev, void* messages_dev,
                 uint64_t* wire_bytes_dev, uint32_t* changed_blocks_dev, void* workspace_dev,
                 int32_t* status_dev, void* stream);

/* ---- sender, for callers that cannot supply scratch ---------------------------------------- */

/* Largest plan ciera_encode_noalloc accepts: 65 536 tiles (ciera_plan_n_tiles), i.e. at most
 * 536 870 912 values per call.  The library keeps 8 bytes per tile (+ 16) = 512 KiB of device memory
 * for it on every GPU that loads the library, from load until the process exits. */
#define CIERA_NOALLOC_MAX_TILES 65536u

/*
 * (This entry point has no counterpart in the paper; it is a convenience of this library.)
 *
 * Same work and same outputs as ciera_encode, but without the `workspace_dev` argument: the
 * look-back scratch is a fixed array inside the library.  It is meant for callers that can pass the
 * buffers they already own but cannot obtain a fresh device allocation when they call -- a training
 * runtime whose memory pool already holds the whole GPU, a parameter-gather hook that must not
 * stall the device (allocating does), a plug-in that was handed pointers but no allocator.  The
 * call itself allocates nothing, on the host or on the device.
 *
 *   - Plans with more than CIERA_NOALLOC_MAX_TILES tiles are refused with CIERA_ERR_TOO_LARGE before
 *     any device work is enqueued; split the unit table, or use ciera_encode with your own scratch.
 *   - The first call on each device looks up the array's device address (a CUDA runtime query made
 *     with that device current).  Make that first call outside of any stream capture.
 *   - All calls on a device share the one array, which keeps whatever the last call left in it; every
 *     call therefore clears the part it uses, on `stream`, before its kernel.  Two calls that can
 *     run on the GPU at the same time (different streams, no ordering between them) race on the
 *     array and produce garbage: order them, or give all but one of them ciera_encode with scratch
 *     of its own.
 */
CIERA_API int ciera_encode_noalloc(const ciera_plan* plan, const void* weights_dev, void* sender_cache_dev,
                         void* messages_dev, uint64_t* wire_bytes_dev, uint32_t* changed_blocks_dev,
                         int32_t* status_dev, void* stream);

/* ---- sender with hash-based change detection (Section 3.1; Algorithm 1, sender, as printed) ---
 *
 * Instead of the previous exponents the sender keeps HashCache: one 128-bit hash per block, built
 * from two independent 64-bit SplitMix64 hashes of the block's exponents.  A block travels iff its
 * hash differs from the cached one; the cached hash is then replaced.  The message is the same as
 * ciera_encode's (a collision -- both 64-bit halves at once, which behave like independent random
 * functions of the block but are not a cryptographic hash -- would leave a changed block unsent).
 * The construction (the paper prints none): with mix() the SplitMix64 output function, a block of L
 * exponent bytes read as little-endian 64-bit words x_j (the last one zero-padded),
 * H_i = mix(L + sum_j mix(s_i + (j + 1) * g_i + x_j)) mod 2^64, Hash128 = (H_1, H_2) with
 * s_1 = 0, g_1 = 0x9E3779B97F4A7C15 (the generator's increment), s_2 = 0x6A09E667F3BCC908,
 * g_2 = 0xD1342543DE82EF95; stored as two little-endian 64-bit words per block.
 * Blocks of 16 values and more only (CIERA_ERR_UNSUPPORTED otherwise).  The hash is taken
 * over the exponents as the caches hold them, one byte each, for every precision. */

/* Bytes of a HashCache for the whole plan (16 per block; units in table order), the offset of a
 * unit's first block in it, and the scratch ciera_encode_hashed needs (= ciera_plan_workspace_bytes). */
CIERA_API size_t ciera_plan_hash_cache_bytes(const ciera_plan* plan);
CIERA_API size_t ciera_plan_unit_hash_offset(const ciera_plan* plan, uint32_t unit);
CIERA_API size_t ciera_plan_hashed_workspace_bytes(const ciera_plan* plan);

/* HashCache := Hash128 of every block of exponents(weights); of all-zero exponents when
 * weights_dev is NULL (the counterpart of a zero-initialised exponent cache).  Device pointers,
 * 16-byte aligned.  Asynchronous on `stream`. */
CIERA_API int ciera_hash_cache_init(const ciera_plan* plan, void* hash_cache_dev, const void* weights_dev, void* stream);

/* Sender step with HashCache.  Arguments, launch (one persistent kernel) and error behaviour as
 * for ciera_encode, with hash_cache_dev (in/out, ciera_plan_hash_cache_bytes) in place of the
 * exponent cache and a scratch of ciera_plan_hashed_workspace_bytes (all zero on entry and on return,
 * as for ciera_encode). */
CIERA_API int ciera_encode_hashed(const ciera_plan* plan, const void* weights_dev, void* hash_cache_dev,
                                  void* messages_dev, uint64_t* wire_bytes_dev, uint32_t* changed_blocks_dev,
                                  void* workspace_dev, int32_t* status_dev, void* stream);

/* ---- transport stand-in: Send / Recv of Algorithm 1 on one GPU ----------------------------- */

/* Copies, for every unit, the first wire_bytes_dev[u] bytes of its slot from `src_messages_dev`
 * to the same slot of `dst_messages_dev` (one kernel; the lengths are read on the device).  This
 * stands where the Allgather of the messages would be.  `workspace_dev`: scratch of
 * ciera_plan_workspace_bytes() (holds the counter tiles are handed out from: zero on entry -- see
 * ciera_workspace_init -- and handed back at zero; not to be shared by calls that can overlap on the GPU).  `status_dev`: device int32 or NULL; the
 * kernel's waits on its own copies are bounded and raise CIERA_ERR_TIMEOUT there. */
CIERA_API int ciera_transport(const ciera_plan* plan, const void* src_messages_dev, void* dst_messages_dev,
                    const uint64_t* wire_bytes_dev, void* workspace_dev, int32_t* status_dev, void* stream);

/* ---- receiver: Algorithm 1, receiver part; Section 3.1 ------------------------------------- */

/*
 * For every unit: read the bitmap, overwrite the cached exponents of changed blocks with the
 * payload, merge cache and sign-plus-mantissa into `weights_out_dev`.
 *   messages_dev        in   slots at units[].msg_off
 *   receiver_cache_dev  i/o  1 byte per value at units[].cache_off
 *   weights_out_dev     out  reconstructed values at units[].weights_off
 *   wire_bytes_dev      in   optional (may be NULL): lengths as reported by the sender; a unit
 *                            whose bitmap implies a different length raises CIERA_ERR_CORRUPT in
 *                            status_dev (its output is then unspecified)
 *   workspace_dev       scratch of ciera_plan_workspace_bytes(), 16-byte aligned: the counter tiles
 *                            are handed out from (zero on entry -- see ciera_workspace_init -- and handed
 *                            back at zero) and, when some unit has
 *                            more than 4096 blocks, the per-tile counts of a small prefix kernel that
 *                            runs first; the sender's part of the workspace is left alone.  Must not be
 *                            shared by calls that can overlap on the GPU.
 */
CIERA_API int ciera_decode(const ciera_plan* plan, const void* messages_dev, void* receiver_cache_dev,
                 void* weights_out_dev, const uint64_t* wire_bytes_dev, void* workspace_dev, int32_t* status_dev,
                 void* stream);

/* ---- whole step ---------------------------------------------------------------------------- */

/*
 * ciera_encode, ciera_transport and ciera_decode of one table in one kernel launch, with the same results: the
 * messages in both buffers, lengths, counts, both caches and the reconstructed weights.  For sender and receiver on
 * one GPU: every byte of a message is stored to both buffers as it is made, and the receiver's part works on it
 * before it leaves the chip, so nothing that the step itself has written is fetched again.  The receiver's weights
 * come from its own cache and the message's contents, as in ciera_decode.
 * Arguments as for the three calls.  One launch needs the buffers apart, but for weights_out_dev, which may be
 * weights_dev; where they overlap in any other way (say, reconstructed weights over the message that was sent), or where
 * units share weights that are reconstructed in place, the call runs the three kernels one after the other.
 */
CIERA_API int ciera_step(const ciera_plan* plan, const void* weights_dev, void* sender_cache_dev, void* msg_send_dev,
                         void* msg_recv_dev, void* receiver_cache_dev, void* weights_out_dev, uint64_t* wire_bytes_dev,
                         uint32_t* changed_blocks_dev, void* workspace_dev, int32_t* status_dev, void* stream);

/* ---- whole step with host buffers ---------------------------------------------------------- */

/* Device buffers one ciera_roundtrip_host call works in; all caller-owned, sized as for the
 * separate calls above (weights_dev / weights_out_dev: weights_bytes each; workspace_dev initialised
 * with ciera_workspace_init as for ciera_encode). */
typedef struct ciera_device_buffers {
    void* weights_dev;
    void* sender_cache_dev;
    void* msg_send_dev;
    void* msg_recv_dev;
    void* receiver_cache_dev;
    void* weights_out_dev;
    uint64_t* wire_bytes_dev;
    uint32_t* changed_blocks_dev;
    void* workspace_dev;
    int32_t* status_dev;
} ciera_device_buffers;

/* One sender + receiver step of Algorithm 1 on weights that live in HOST memory:
 * copy `weights_host` (weights_bytes, ideally pinned) to the device, step as ciera_step does, copy the
 * reconstructed weights to `weights_out_host` (which may be or overlap `weights_host`) and the per-unit wire
 * lengths to `wire_bytes_host` ([n_units], may be NULL).
 *   - Pinned weights of 4 MB and more are stepped in parts, so that the host link carries both directions at
 *     once: the copies run on streams of the library, between what `stream` held before and what it is given
 *     next, and a part is one kernel launch on `stream`.  Pageable memory, and a stream that is being captured:
 *     as a whole, all on `stream`.
 *   - The host buffers must stay valid until `stream` has drained.
 *   - Any number of threads and streams may step at the same time, each with buffers of its own.
 *   - If a copy to the device cannot be queued, nothing is stepped; if one back cannot, the step on the device
 *     is complete.  After any other CUDA error the caches may hold the exponents of some tiles already; the
 *     workspace can be used again in every case. */
CIERA_API int ciera_roundtrip_host(const ciera_plan* plan, const void* weights_host, size_t weights_bytes,
                         void* weights_out_host, uint64_t* wire_bytes_host, const ciera_device_buffers* bufs,
                         void* stream);

/* ---- entropy stage (Section 3.1; Algorithm 1: ANSEncode on the sender, ANSDecode on the receiver) ---
 *
 * Between ciera_encode (or ciera_encode_hashed) and the transport, ciera_entropy_encode replaces the
 * payload of every message -- the exponents of the changed blocks -- by its rANS-coded form if that
 * is strictly shorter, and lowers the unit's wire_bytes accordingly; bitmap and sign-plus-mantissa
 * stay as they are.  Between the transport and ciera_decode, ciera_entropy_decode restores the raw
 * payload in place (the receiver knows the raw length from the bitmap: a message of exactly that
 * length carries the raw form) and sets wire_bytes back to the raw length, so that ciera_decode
 * sees what the sender step had written.  The paper names a vendor library whose format is not
 * public; coder and layout are this library's own: static model per unit (a symbol = an exponent:
 * 256 symbols for bf16 and fp32, 32 for fp16, whose 5-bit packing is undone before and redone after
 * the coder; probabilities in 1/4096), 32-bit rANS states with 16-bit words, segments of 4096
 * symbols coded by 32 interleaved coders each; coded section = [256 or 32 x u16 frequencies][per
 * segment a u32 word count][segments: 32 x u32 final states, the words, 2 zero bytes if their
 * number is odd].
 *   messages_dev    device, in/out
 *   wire_bytes_dev  device, n_units x uint64, in/out
 *   scratch_dev     device, ciera_plan_entropy_scratch_bytes(plan) bytes, 16-byte aligned; contents
 *                   need not be initialised
 *   status_dev      device int32 or NULL: CIERA_ERR_CORRUPT if a coded section is inconsistent
 *                   (that unit's payload is then left as received)
 * One launch each for short units, a thread block per unit; longer units are cut into chunks of 64 segments, which
 * takes up to six launches more (decode: three).  Nothing waits inside the kernels. */
CIERA_API size_t ciera_plan_entropy_scratch_bytes(const ciera_plan* plan);
CIERA_API int ciera_entropy_encode(const ciera_plan* plan, void* messages_dev, uint64_t* wire_bytes_dev, void* scratch_dev,
                                   void* stream);
CIERA_API int ciera_entropy_decode(const ciera_plan* plan, void* messages_dev, uint64_t* wire_bytes_dev, void* scratch_dev,
                                   int32_t* status_dev, void* stream);

/* ---- selective compression: the gain rule of Section 3.2 (host only) ----------------------- */

typedef struct ciera_gain_in {
    uint64_t n_values;    /* N^i                                                               */
    int32_t dtype;        /* ciera_dtype                                                        */
    uint32_t block;       /* B (any positive value; only sizes are computed)                    */
    double q;             /* block change rate q_i in [0, 1] (measured offline / by a previous encode) */
    int32_t world_size;   /* W, used by the alpha-beta model only                               */
    int32_t overlapped;   /* non-zero: T_hash = T_cmp = 0 on the critical path (pipelining)     */
    double alpha;         /* Comm(S) = alpha + (W-1) * S / beta when n_points < 2               */
    double beta;          /* bytes per second                                                   */
    const double* table_bytes; /* optional measured Comm(): n_points ascending payload sizes... */
    const double* table_secs;  /* ...and their latencies; linear interpolation, the first/last
                                  segment is extended outside the table                         */
    int32_t n_points;
    double t_hash;        /* seconds: change detection of the shard                             */
    double t_cmp;         /* seconds: sender-side packing                                       */
    double t_decmp;       /* seconds: receiver-side patch + merge                               */
} ciera_gain_in;

/* g = Comm(S) - ( Comm(S_{s+m} + S_bm + q S_e) + T_hash + T_cmp + T_decmp ), and the decision
 * "compress iff g > 0".  Either output pointer may be NULL. */
CIERA_API int ciera_should_compress(const ciera_gain_in* in, double* gain_seconds_out, int* decision_out);

/* Shard selection under a cache budget (Section 3.2, last paragraph): shard i costs
 * M_i = (W - 1) * S_e^i bytes of exponent cache per GPU (S_e^i = one byte per value); shards with
 * positive gain are ranked in descending order of g_i / M_i and selected down the ranking until the
 * first one that no longer fits into cache_budget_bytes (ties keep the input order; shards without
 * values are never selected).  with_sender_cache != 0 counts W * S_e^i instead, i.e. also the
 * sender-side exponent cache this library compares against.
 *   shards          host, n_shards entries (q_i, sizes, Comm() model and kernel times per shard)
 *   ranking_out     host, n_shards indices: the ranked positive-gain shards, then the others in
 *                   input order; may be NULL
 *   selected_out    host, n_shards flags (1 = compress this shard)
 *   gains_out, footprints_out   host, n_shards values g_i (seconds) and M_i (bytes); may be NULL
 *   used_bytes_out  host, sum of M_i over the selected shards; may be NULL
 * Returns CIERA_ERR_INVALID_ARG for a shard that ciera_should_compress would reject. */
CIERA_API int ciera_select_shards(const ciera_gain_in* shards, uint32_t n_shards, uint64_t cache_budget_bytes,
                                  int with_sender_cache, uint32_t* ranking_out, uint8_t* selected_out,
                                  double* gains_out, uint64_t* footprints_out, uint64_t* used_bytes_out);

/* ---- the MoE layer behind the gather ---------------------------------------------------------- */

/* What the gathered experts are needed for (no counterpart in the paper, which leaves the layer to the training
 * framework): tokens are routed to experts, their rows laid out expert by expert, multiplied with the experts'
 * matrices in 8-bit floating point, and summed back.  All calls only enqueue work on `stream`, read every size that
 * depends on the routing on the device, keep nothing between calls, and give the same bits for the same inputs.
 * dtype arguments are ciera_dtype values; strides count elements; every tensor's last dimension is contiguous.  Buffers
 * of one call do not overlap.  Base pointers of 16-, 32- and 64-bit data are aligned to one value; wider alignment is
 * used where it is there. */

typedef enum ciera_score { CIERA_SCORE_SOFTMAX = 0, CIERA_SCORE_SIGMOID = 1 } ciera_score;

/* Routing.  For each token with logits l[0 .. n_experts):
 *   s = softmax(l) or, value by value, sigmoid(l);   c = s + bias (bias 0 if NULL)
 *   an expert whose logit is -inf or NaN, or whose c is -inf or NaN, is closed: its s is 0 where the logit closes it,
 *   and it is never chosen; +inf counts as the largest finite number, -0 as 0
 *   groups of n_experts / n_groups neighbours; a group's value is the sum of its `group_best` (1 or 2) largest c; the
 *   top_groups groups of the largest values stay (a group without an open expert never does)
 *   the top_k largest c among them are chosen, in falling order; equal values go to the lower index
 *   w = scale * s of the chosen, divided by the sum of their s if `renormalise` (0 where that sum is 0 in 64 bits)
 * Choices are those of 64-bit arithmetic, and so are quotients by a sum below 1e-10; other weights are 32-bit arithmetic.  Where fewer than top_k experts are open, the rest has index -1 and weight 0.
 * Limits: n_experts 1 .. 1024, top_k 1 .. 32 and at most top_groups * (n_experts / n_groups), n_groups 1 .. 32 and a
 * divisor of n_experts, scale finite. */
typedef struct ciera_route_config {
    uint32_t n_experts, top_k, n_groups, top_groups, group_best;
    int32_t score;       /* ciera_score */
    int32_t renormalise; /* 0 or 1 */
    float scale;
} ciera_route_config;

/*   logits   device, n_tokens rows of n_experts values, logits_stride apart
 *   bias     device, n_experts fp32, or NULL: added for the choice only
 *   experts  device, n_tokens x top_k int32;  weights  device, n_tokens x top_k fp32 */
CIERA_API int ciera_route(const ciera_route_config* config, int dtype, const void* logits_dev, uint64_t n_tokens,
                          uint64_t logits_stride, const float* bias_dev, int32_t* experts_dev, float* weights_dev,
                          void* stream);
/* Gradient of the logits from that of the weights, for the choice in `experts` (entries outside 0 .. n_experts - 1 and
 * their dweights are passed over).  Through the scores and, if asked for, the renormalisation; the choice and the bias
 * have none.  Closed experts get 0.  dlogits has the logits' type; every value of its rows is written. */
CIERA_API int ciera_route_backward(const ciera_route_config* config, int dtype, const void* logits_dev, uint64_t n_tokens,
                                   uint64_t logits_stride, const int32_t* experts_dev, const float* dweights_dev,
                                   void* dlogits_dev, uint64_t dlogits_stride, void* stream);

/* Rows of a segment are a multiple of this, and so many values share a scale. */
#define CIERA_FP8_BLOCK 128

/* Layout of n_slots slots (token * top_k + choice) by expert: expert e's slots in rising order at rows starts[e] ..
 * starts[e] + counts[e] - 1, its segment ends at starts[e + 1], a multiple of 128.  Slots whose expert is outside
 * 0 .. n_experts - 1 get no row (-1).
 *   starts       device, n_experts + 1 int32;  counts  device, n_experts int32
 *   row_of_slot  device, n_slots int32
 *   slot_of_row  device, ciera_expert_rows_capacity() int32: -1 for the rows that fill a segment up; rows from
 *                starts[n_experts] on are left as they were
 *   workspace    device, ciera_expert_layout_workspace_bytes(); any contents, not shared by calls that may overlap
 * Limits: n_experts 1 .. 1024, at most 2^30 slots. */
CIERA_API uint64_t ciera_expert_rows_capacity(uint64_t n_slots, uint32_t n_experts);
CIERA_API size_t ciera_expert_layout_workspace_bytes(uint64_t n_slots, uint32_t n_experts);
CIERA_API int ciera_expert_layout(const int32_t* experts_dev, uint64_t n_slots, uint32_t n_experts, int32_t* starts_dev,
                                  int32_t* counts_dev, int32_t* row_of_slot_dev, int32_t* slot_of_row_dev, void* workspace,
                                  void* stream);

/* Operands in e4m3 (finite, largest 448) with a power of two for each block of 128 values.  With the block's largest
 * magnitude a, s is the least integer >= -126 with a <= 448 * 2^s (0 for a block of zeros); the scale byte is s + 127 and
 * stands for 2^s; a value y is stored as y * 2^-s rounded to nearest, ties to even.  A block that holds an infinity or a
 * NaN has byte 255 and NaN in all its places.
 * Scale bytes of an operand [rows, cols] whose blocks lie along the columns: byte (column / 128) * stride + row. */
typedef enum ciera_fp8_source {
    CIERA_SOURCE_ROWS = 0,           /* y = x, or x of the row's token (slot_of_row), or row_weights[slot] * that           */
    CIERA_SOURCE_SWIGLU = 1,         /* y[:, j] = silu(x[:, j]) * x[:, cols + j]; x has 2 * cols columns                     */
    CIERA_SOURCE_SWIGLU_BACKWARD = 2 /* gradient of that by x: cols even, x has cols columns, grad has cols / 2              */
} ciera_fp8_source;

/* Rows of an operand, formed from `x` and rounded in one pass.
 *   q, scales      blocks along the columns: q [rows, cols], ceil(cols / 128) rows of scale bytes
 *   qt, scales_t   or NULL, NULL: the same y transposed, blocks of 128 rows: qt [cols, rows], ceil(rows / 128) rows of
 *                  scale bytes (one for each column of y)
 *   slot_of_row    or NULL.  With CIERA_SOURCE_ROWS row r is made from x's row slot_of_row[r] / top_k; with the others
 *                  from x's row r.  Rows without a slot (negative, or beyond x_rows * top_k) are zero.
 *   row_weights    or NULL; x_rows * top_k fp32 (CIERA_SOURCE_ROWS with slot_of_row only)
 *   starts         or NULL: rows from starts[n_experts] on are left as they were, in q, qt and the scales alike
 * q and qt are 16-byte aligned with strides that are multiples of 16 and at least cols / rows.  Limits: rows and cols
 * 1 .. 2^31 - 256.  Arithmetic in 32 bits (in 64 for gates below -87, where sigmoid leaves 32 bits); the scale is that of
 * 64-bit arithmetic where silu stands in between. */
typedef struct ciera_fp8_rows {
    int32_t source, dtype; /* dtype of x and grad */
    uint64_t rows, cols, x_rows;
    const void* x;
    uint64_t x_stride;
    const void* grad;
    uint64_t grad_stride;
    const int32_t* slot_of_row;
    const float* row_weights;
    const int32_t* starts;
    uint32_t top_k, n_experts;
    void* q;
    uint64_t q_stride;
    uint8_t* scales;
    uint64_t scales_stride;
    void* qt;
    uint64_t qt_stride;
    uint8_t* scales_t;
    uint64_t scales_t_stride;
} ciera_fp8_rows;
CIERA_API int ciera_fp8_quantize_rows(const ciera_fp8_rows* args, void* stream);

/* Matrices with one scale for each block of 128 x 128: x is `matrices` matrices [rows, cols], x_stride between rows,
 * x_matrix_stride between matrices.  scales: byte (matrix, row / 128, column / 128) at matrix * scales_matrix_stride +
 * (row / 128) * scales_stride + column / 128.  qt, scales_t (or NULL, NULL): the transposed matrices [cols, rows]. */
typedef struct ciera_fp8_blocks {
    int32_t dtype;
    uint32_t matrices;
    uint64_t rows, cols;
    const void* x;
    uint64_t x_stride, x_matrix_stride;
    void* q;
    uint64_t q_stride, q_matrix_stride;
    uint8_t* scales;
    uint64_t scales_stride, scales_matrix_stride;
    void* qt;
    uint64_t qt_stride, qt_matrix_stride;
    uint8_t* scales_t;
    uint64_t scales_t_stride, scales_t_matrix_stride;
} ciera_fp8_blocks;
CIERA_API int ciera_fp8_quantize_blocks(const ciera_fp8_blocks* args, void* stream);

/* Products of such operands, out = sum over blocks of 2^(sa + sb) * (a_block * b_block^T), summed in fp32.
 *   CIERA_PRODUCT_DENSE     out [m, n] = a [m, k] * b [n, k]^T
 *   CIERA_PRODUCT_ROWS      rows starts[e] .. starts[e + 1] - 1 of a and out with matrix e of b [n_experts][n, k]; rows of
 *                           out from starts[n_experts] on are left as they were
 *   CIERA_PRODUCT_CONTRACT  out [n_experts][m, n]: a [m, k] * b [n, k]^T over the columns starts[e] .. starts[e + 1] - 1
 *                           alone; zeros for an empty segment
 * a has a scale for each row and 128 columns; b the same (b_blocks 0, CONTRACT and DENSE) or one for each block of
 * 128 x 128 (b_blocks 1, DENSE and ROWS; strides as in ciera_fp8_blocks).
 * starts rise from 0, are multiples of 128 and end at or below m (ROWS) or k (CONTRACT): otherwise CIERA_ERR_CORRUPT is
 * written to *status, if given, and no output; CIERA_ERR_TIMEOUT if a bounded device wait ran out.  a, b are 16-byte aligned,
 * their strides multiples of 16 and at most 2^40 - 16.  Where lines of scale bytes start at multiples of 4, the rest of an
 * aligned word that holds a row's byte may be read with it, and is not used.  Limits: m, n, k 1 .. 2^31 - 256, n_experts
 * 1 .. 1024. */
typedef enum ciera_product_mode {
    CIERA_PRODUCT_DENSE = 0,
    CIERA_PRODUCT_ROWS = 1,
    CIERA_PRODUCT_CONTRACT = 2
} ciera_product_mode;
typedef struct ciera_fp8_product {
    int32_t mode, out_dtype, b_blocks;
    uint32_t n_experts;
    uint64_t m, n, k;
    const void* a;
    uint64_t a_stride;
    const uint8_t* a_scales;
    uint64_t a_scales_stride;
    const void* b;
    uint64_t b_stride, b_matrix_stride;
    const uint8_t* b_scales;
    uint64_t b_scales_stride, b_scales_matrix_stride;
    const int32_t* starts;
    void* out;
    uint64_t out_stride, out_matrix_stride;
    int32_t* status;
} ciera_fp8_product;
CIERA_API int ciera_fp8_matmul(const ciera_fp8_product* args, void* stream);

/* Weighted sum of a token's rows: out[t] = sum over j of weights[t, j] * rows[row_of_slot[t, j]], in fp32, rounded once;
 * weights NULL: 1.  Entries of row_of_slot outside 0 .. n_rows - 1 are passed over (a token without any gets zeros).
 *   rows  device, n_rows rows of `cols` values of `dtype`;  out  device, n_tokens rows, same type
 * Limits: top_k 1 .. 32, cols 1 .. 2^31 - 256, n_tokens * top_k and n_rows up to 2^31 - 256. */
CIERA_API int ciera_expert_combine(int dtype, const void* rows_dev, uint64_t n_rows, uint64_t rows_stride,
                                   const int32_t* row_of_slot_dev, const float* weights_dev, uint64_t n_tokens,
                                   uint32_t top_k, uint64_t cols, void* out_dev, uint64_t out_stride, void* stream);
/* Its gradients from that of out: dweights[t, j] = sum of dout[t] * rows[row] in fp32 (0 for entries passed over), and,
 * if drows is given, drows[row] = weights[t, j] * dout[t] (rows that no entry names are left as they were; entries name
 * different rows). */
CIERA_API int ciera_expert_combine_backward(int dtype, const void* dout_dev, uint64_t dout_stride, const void* rows_dev,
                                            uint64_t n_rows, uint64_t rows_stride, const int32_t* row_of_slot_dev,
                                            const float* weights_dev, uint64_t n_tokens, uint32_t top_k, uint64_t cols,
                                            float* dweights_dev, void* drows_dev, uint64_t drows_stride, void* stream);

/* ---- diagnostics ---------------------------------------------------------------------------- */

/* Self-test of the device-side failure path (no counterpart in the paper: Algorithm 1 has no failure
 * handling).  Every wait inside the persistent kernels -- on a look-back status word of another tile,
 * on a shared-memory barrier that a bulk copy or another warp completes -- is bounded: when the bound
 * runs out the waiting role raises CIERA_ERR_TIMEOUT in the caller's status word, the thread block
 * stops, and the kernel returns, so the context stays usable.  This call runs one tiny kernel (one
 * thread block) that performs both kinds of wait with a limit of `max_polls` polls (1 .. 4096; a
 * barrier poll suspends for at most 20 microseconds) on a word and a barrier that nothing completes.
 *   scratch_dev  device, 8 bytes, 8-byte aligned: the status word that is polled (cleared by the call)
 *   status_dev   device int32: receives CIERA_ERR_TIMEOUT if it was 0
 *   report_dev   device, 4 x int32 (cleared by the call): [0] = 1 the status-word wait gave up,
 *                [1] = 1 the barrier wait gave up, [2] = the block's abort flag, [3] = max_polls
 * Asynchronous on `stream`. */
CIERA_API int ciera_selftest_bounded_waits(uint32_t max_polls, void* scratch_dev, int32_t* status_dev,
                                           int32_t* report_dev, void* stream);

/* cudaError_t of the last failing runtime call made by the calling thread inside this library. */
CIERA_API int ciera_last_cuda_error(void);
/* Number of kernels this library has launched from the calling process (for launch accounting). */
CIERA_API uint64_t ciera_kernel_launch_count(void);
CIERA_API const char* ciera_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* CIERA_H */
