// A whole MoE layer for a few tokens.
//
// What it costs is reading the matrices of the experts that are reached, once: one token of 8 experts of 2048 x 1024 reads 50 MB
// in 8 bits and multiplies each weight once.  So the weights go from memory to the tensor cores without passing through a
// register: a tile of 128 rows comes by tensor map and is the first operand as it is, in 8 bits (kind::mxf8f6f4) or 4 (kind::mxf4),
// with its powers of two; the tokens are the second operand, in the same bits.  A token's values are not rounded to those: they come as
// a sum of parts, each rounded to 8 or 4 bits below a power of two of its own for 32 values, every part a column of the product,
// whose sums are added in the end.  An e4m3 part has four bits and a sign, so five take all 24 of a 32-bit value, x's or the middle's.  An
// e2m1 part takes three bits below the largest of 32: seven leave 2^-19 of that at most, what rounding a value 2^10 times smaller to bf16
// does, and nine (fp32) 2^-25.  (Three and six, 2^-14 of a value and 2^-13 of the largest: 64 tokens in 8 bits 72.1 us, 73.9 so;
// 34 of 128 experts of 256 x 1920 47.6, 57.9; in 4 bits 64 tokens 51.1, 52.4.  Nine in 4 bits for all types: 56.5.)
// (With weights made fp16 in registers and 16-bit tensor products the same took 300 instructions for 2 KB: one token 24 us, 64
// tokens 164 us.)
//
// One kernel behind the router's, whose blocks all run at once (a cooperative launch):
//   parts  the tokens' rows as parts, while the router still runs
//   up     tiles of 64 rows of the gate and the same 64 of up; silu(g) * u goes to the workspace as parts again
//   down   tiles of 128 rows of the output, expert by expert, as fp32 to the workspace
//   sum    a token's rows, weighted, in the order of its choices
// What one part reads of another's results, only the copies of the second operand wait for: those of the weights go on, so that a
// block's next 96 to 160 KB of them are on their way meanwhile.  A tile of down waits for its group's tiles of up, which were the
// first to be made (for all of up: 64 tokens 76 us, 72 so).
// Tokens of an expert are taken 16 at a time (a group; 12 where there are nine parts): 112 columns.
#include <type_traits>

#include "ciera_fp4.cuh"
#include "ciera_fp8.cuh"
#include "ciera_product.cuh"
#include "ciera_route.cuh"
#include "ciera_swiglu.cuh"
#include "ciera_tokens_end.hpp"

namespace ciera {

constexpr int kTokenThreads = 384, kTokenWarps = kTokenThreads / 32;
constexpr uint32_t kColumnWarps = 4;  // that copy the tokens' columns, a stage each in turn
constexpr int kMostStages = 10;
constexpr int kBehind = 5;  // stages whose weights' scales are on their way; fewer than there are stages
constexpr uint32_t kMaxSlots = CIERA_EXPERT_TOKENS_MAX * 32;
constexpr uint32_t kMaxColumns = 112;
constexpr uint32_t kMaxReportPolls = 1u << 25;  // of some tens of ns: longer than what is waited for may take
constexpr uint32_t kTokenHead = CIERA_EXPERT_TOKENS_HEAD;  // bytes of the workspace's counters
static_assert(kTokenHead >= 256 + 4 * kMaxSlots, "a counter for each group");
constexpr uint32_t kTileBytes = 128 * 128;
// Tensor memory: two sums, and the scales of more stages than the ring has, so that the products of a stage whose place a later one's
// scales take have ended when that one has come.  (Four or two stages' scales, and a wait for them: 0.5 us a call.)
constexpr uint32_t kSumColumns = 112, kTokenScalesAt = 2 * kSumColumns, kTokenTmem = 512;
constexpr uint32_t kScaleBuffers = 16;
static_assert(kScaleBuffers > kMostStages && kTokenScalesAt + kScaleBuffers * 16 <= kTokenTmem, "not in tensor memory");

// Parts of a value and slots of a group.
template <int BITS, int DT>
constexpr int kParts = BITS == 8 ? 5 : DT == CIERA_FP32 ? 9 : 7;
template <int BITS, int DT>
constexpr uint32_t kGroupSlots = kMaxColumns / kParts<BITS, DT> < 16 ? kMaxColumns / kParts<BITS, DT> : 16;

struct Matrices {
    const uint8_t* scales;
    uint64_t scales_stride, scales_matrix_stride;
};
struct TokensArgs {
    Matrices w1, w2;
    const int32_t* experts;
    const float* weights;
    uint64_t x_stride, out_stride;
    uint32_t* counters;  // blocks that are done with parts, tiles of up, blocks done with down, with all; from 64 on each group's tiles of
                         // up.  Zero before and after
    int32_t* status;
    uint8_t* x_parts;        // [tokens * parts][d_model], 8 or 4 bits
    uint32_t* x_scales;      // [d_model / 128][tokens * parts]
    uint8_t* hidden;         // [slots * parts][d_ff]
    uint32_t* hidden_scales;
    float* rows;             // [slots][d_model]
    uint32_t n_tokens, top_k, n_experts, d_model, d_ff;
    uint32_t stages, stage_bytes;
    int32_t x_wide, out_wide;  // four values at a time
};

// The slots of the reached experts in the order of the experts, each at a place, and groups of up to `most` of an expert's.
struct TokenLists {
    uint32_t group[kMaxSlots];   // expert << 16 | slots - 1 << 11 | first place
    uint16_t place[kMaxSlots];   // of a slot; 0xffff: none
    uint8_t token[kMaxSlots];    // at a place
    uint32_t warp_total[kTokenWarps];
    uint32_t groups;
};
struct ListScratch {
    uint32_t at[1024];  // first place of an expert
    uint16_t count[kMaxSlots / 32 * 1024];  // [32 slots][expert], n_experts apart: the expert's slots; then those before
};
__device__ __forceinline__ uint32_t group_expert(uint32_t g) { return g >> 16; }
__device__ __forceinline__ uint32_t group_slots(uint32_t g) { return (g >> 11 & 31u) + 1; }
__device__ __forceinline__ uint32_t group_first(uint32_t g) { return g & 2047u; }

// By the whole block; ends with a barrier.
__device__ __forceinline__ void make_lists(TokenLists& l, ListScratch& s, const TokensArgs& a, uint32_t most) {
    const uint32_t n = a.n_tokens * a.top_k, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.n_experts;
    if (n <= 32) {  // by one warp, a slot a lane
        if (warp == 0) {
            const int32_t id = lane < n ? __ldcg(a.experts + lane) : -1;
            const uint32_t e = (uint32_t)id < E ? (uint32_t)id : 0xffffu;
            uint32_t place = 0, rank = 0, count = 0, groups = 0;  // places before, before of the same expert, the expert's, groups before
            for (uint32_t i = 0; i < n; ++i) {
                const uint32_t o = __shfl_sync(~0u, e, i);
                place += o < e || (o == e && i < lane);
                rank += o == e && i < lane;
                count += o == e;
            }
            const bool first = rank % most == 0 && e != 0xffffu;  // the lane makes a group
            for (uint32_t i = 0; i < n; ++i) groups += __shfl_sync(~0u, first ? place : ~0u, i) < place;
            if (lane < n) l.place[lane] = (uint16_t)(e == 0xffffu ? 0xffffu : place);
            if (e != 0xffffu) l.token[place] = (uint8_t)(lane / a.top_k);
            if (first) l.group[groups] = e << 16 | (min(most, count - rank) - 1) << 11 | place;
            const uint32_t all = __popc(__ballot_sync(~0u, first));
            if (lane == 0) l.groups = all;
        }
        __syncthreads();
        return;
    }
    // slots of an expert are counted for each 32 neighbours, then over those before
    constexpr int kEach = (kMaxSlots + kTokenThreads - 1) / kTokenThreads;
    const uint32_t chunks = (n + 31) / 32;
    for (uint32_t i = tid; i < (chunks * E + 7) / 8; i += kTokenThreads) reinterpret_cast<uint4*>(s.count)[i] = make_uint4(0, 0, 0, 0);
    int32_t id[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t i = j * kTokenThreads + tid;
        id[j] = i < n ? __ldcg(a.experts + i) : -1;
        if ((uint32_t)id[j] >= E) id[j] = -1;
    }
    __syncthreads();
    uint32_t rank[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t chunk = j * kTokenWarps + warp;
        if (chunk >= chunks) break;
        const uint32_t same = __match_any_sync(~0u, id[j]);
        rank[j] = __popc(same & ((1u << lane) - 1));
        if (id[j] >= 0 && rank[j] == 0) s.count[chunk * E + id[j]] = (uint16_t)__popc(same);
    }
    __syncthreads();
    // an expert's slots before each 32, then places and groups before each expert, a thread for each (of 384 at a time): slots in the
    // low half, groups in the high one
    uint32_t base = 0;
    for (uint32_t e0 = 0; e0 < E; e0 += kTokenThreads) {
        const uint32_t e = e0 + tid;
        uint32_t count = 0;
        if (e < E)
#pragma unroll 4
            for (uint32_t c = 0; c < chunks; ++c) {
                const uint32_t v = s.count[c * E + e];
                s.count[c * E + e] = (uint16_t)count;
                count += v;
            }
        const uint32_t v = count | (count + most - 1) / most << 16;
        uint32_t sum = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(~0u, sum, d);
            if (lane >= (uint32_t)d) sum += o;
        }
        if (lane == 31) l.warp_total[warp] = sum;
        __syncthreads();
        uint32_t before = base;
#pragma unroll
        for (uint32_t w = 0; w < kTokenWarps; ++w) {
            const uint32_t o = l.warp_total[w];
            if (w < warp) before += o;
            base += o;
        }
        before += sum - v;
        uint32_t g = before >> 16;
        const uint32_t at = before & 0xffffu;
        for (uint32_t c = 0; c < count; c += most, ++g) l.group[g] = e << 16 | (min(most, count - c) - 1) << 11 | (at + c);
        if (e < E) s.at[e] = at;
        __syncthreads();
    }
    if (tid == 0) l.groups = base >> 16;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t chunk = j * kTokenWarps + warp, slot = j * kTokenThreads + tid;
        if (chunk >= chunks) break;
        uint32_t place = 0xffffu;
        if (id[j] >= 0) {
            place = s.at[id[j]] + s.count[chunk * E + id[j]] + rank[j];
            l.token[place] = (uint8_t)(slot / a.top_k);
        }
        if (slot < n) l.place[slot] = (uint16_t)place;
    }
    __syncthreads();
}

// ---- parts

// The scale byte of 32 values whose largest magnitude has these bits, and what takes them below it (0 where they are not finite).
template <int BITS>
__device__ __forceinline__ uint32_t part_byte(uint32_t amax) {
    return BITS == 8 ? scale_byte(amax) : scale_byte4(amax);
}
__device__ __forceinline__ float part_inverse(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }

// Four values rounded to e4m3, and what is left of them.
__device__ __forceinline__ uint32_t take_part8(float (&v)[4], float inv, float unit) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0] * inv, v[1] * inv), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2] * inv, v[3] * inv), __NV_SATFINITE, __NV_E4M3);
    const float2 a = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)lo, __NV_E4M3)));
    const float2 b = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)hi, __NV_E4M3)));
    v[0] = fmaf(-a.x, unit, v[0]);
    v[1] = fmaf(-a.y, unit, v[1]);
    v[2] = fmaf(-b.x, unit, v[2]);
    v[3] = fmaf(-b.y, unit, v[3]);
    return lo | hi << 16;
}
// Four values rounded to e2m1 in 16 bits, and what is left of them.
__device__ __forceinline__ uint32_t take_part4(float (&v)[4], float inv, float unit) {
    uint32_t r, ab, cd;
    asm("{\n\t.reg .b8 a, b, n;\n\t.reg .b16 z;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %6, %5;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b;\n\t"
        "mov.b16 z, 0;\n\tcvt.u8.u16 n, z;\n\t"
        "mov.b32 %0, {a, b, n, n};\n\t}"
        : "=r"(r), "=r"(ab), "=r"(cd)
        : "f"(v[0] * inv), "f"(v[1] * inv), "f"(v[2] * inv), "f"(v[3] * inv));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&ab)), b = __half22float2(*reinterpret_cast<const __half2*>(&cd));
    v[0] = fmaf(-a.x, unit, v[0]);
    v[1] = fmaf(-a.y, unit, v[1]);
    v[2] = fmaf(-b.x, unit, v[2]);
    v[3] = fmaf(-b.y, unit, v[3]);
    return r;
}

// What a part leaves fits below a power of two that is known beforehand, so only the first part's has to be looked for.  Of values up to
// 448 * 2^s e4m3 leaves at most 16 * 2^s = 256 * 2^(s - 4), and of those up to 256 units 8, which is 256 of a unit 32 times smaller.  Of
// values up to 6 * 2^s e2m1 leaves at most 2^s = 4 * 2^(s - 2), and of those up to 4 units 1/2, which is 4 of a unit 8 times smaller.
// (A reduction over 32 lanes for each part: 1 us for the six of one slot, of which a tile has up to 16.)
template <int BITS>
__device__ __forceinline__ uint32_t next_byte(uint32_t first, uint32_t p) {
    const int below = p == 0 ? 0 : BITS == 8 ? 4 + 5 * (int)(p - 1) : 2 + 3 * (int)(p - 1);
    return (uint32_t)max((int)first - below, 1);
}

// 128 values of a token, four a lane, as parts.
template <int DT, int BITS>
__device__ __forceinline__ void make_parts(const TokensArgs& a, const value_t<DT>* x, uint32_t token, uint32_t kb, uint32_t lane) {
    constexpr uint32_t P = kParts<BITS, DT>;
    float v[4];
    const value_t<DT>* from = x + token * a.x_stride + kb * 128 + lane * 4;
    if (a.x_wide) {
        load_values<DT, 4>(from, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ValueOf<DT>::get(from[i]);
    }
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) amax = max(amax, __shfl_xor_sync(~0u, amax, d));
    uint32_t first = part_byte<BITS>(amax);
    const bool bad = first == 255u;  // NaN by its first part's scale; the rest is zeros
    if (bad) {
        first = 127u;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0.f;
    }
    uint32_t own = 0;  // lane p: the four groups' bytes of part p
#pragma unroll
    for (uint32_t p = 0; p < P; ++p) {
        const uint32_t byte = next_byte<BITS>(first, p), row = token * P + p;
        const float inv = part_inverse(byte), unit = __uint_as_float(byte << 23);
        if constexpr (BITS == 8) *reinterpret_cast<uint32_t*>(a.x_parts + (uint64_t)row * a.d_model + kb * 128 + lane * 4) = take_part8(v, inv, unit);
        else *reinterpret_cast<uint16_t*>(a.x_parts + (uint64_t)row * (a.d_model / 2) + kb * 64 + lane * 2) = (uint16_t)take_part4(v, inv, unit);
        uint32_t all = (p == 0 && bad ? 255u : byte) << (lane >> 3) * 8;
        all |= __shfl_xor_sync(~0u, all, 8);
        all |= __shfl_xor_sync(~0u, all, 16);
        if (lane == p) own = all;
    }
    if (lane < P) a.x_scales[(uint64_t)kb * (a.n_tokens * P) + token * P + lane] = own;
}

// 32 neighbouring values of the middle, one a lane, as parts at one place; columns f ... of d_ff.
template <int DT, int BITS>
__device__ __forceinline__ void put_hidden(const TokensArgs& a, float v, uint32_t place, uint32_t f, uint32_t lane) {
    constexpr uint32_t P = kParts<BITS, DT>;
    const uint32_t rows = a.n_tokens * a.top_k * P;
    uint32_t first = part_byte<BITS>(__reduce_max_sync(~0u, __float_as_uint(v) & 0x7fffffffu));
    const bool bad = first == 255u;
    if (bad) first = 127u, v = 0.f;
    if (lane < P)
        reinterpret_cast<uint8_t*>(a.hidden_scales + (uint64_t)(f >> 7) * rows + place * P + lane)[f >> 5 & 3u] =
            (uint8_t)(lane == 0 && bad ? 255u : next_byte<BITS>(first, lane));
    if constexpr (BITS == 8) {
        uint8_t* to = a.hidden + (uint64_t)place * P * a.d_ff + f + lane;
#pragma unroll
        for (uint32_t p = 0; p < P; ++p) {
            const uint32_t byte = next_byte<BITS>(first, p);
            const uint8_t q = __nv_cvt_float_to_fp8(v * part_inverse(byte), __NV_SATFINITE, __NV_E4M3);
            v = fmaf(-__half2float(__half(__nv_cvt_fp8_to_halfraw(q, __NV_E4M3))), __uint_as_float(byte << 23), v);
            to[(uint64_t)p * a.d_ff] = q;
        }
    } else {  // an even lane has its neighbour's value too
        const float other = __shfl_down_sync(~0u, v, 1);
        if (lane & 1) return;
        float pair[4] = {v, other, 0.f, 0.f};
        uint8_t* to = a.hidden + (uint64_t)place * P * (a.d_ff / 2) + (f + lane) / 2;
#pragma unroll
        for (uint32_t p = 0; p < P; ++p) {
            const uint32_t byte = next_byte<BITS>(first, p);
            to[(uint64_t)p * (a.d_ff / 2)] = (uint8_t)take_part4(pair, part_inverse(byte), __uint_as_float(byte << 23));
        }
    }
}

// ---- tensor cores of one block (ciera_tensor.cuh has the pair's)

__device__ __forceinline__ void tmem_alloc_one(uint32_t* where, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_one(uint32_t at, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tensor_commit_one(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_copy_scales_one(uint32_t to, uint64_t rows) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(rows) : "memory");
}
template <int BITS>
__device__ __forceinline__ void tensor_mma_one(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t a_scales, uint32_t b_scales, bool add) {
    if constexpr (BITS == 8)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(instruction), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(instruction), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add)
            : "memory");
}
__device__ __forceinline__ void map_load3_one(void* dst, const void* map, int32_t x, int32_t y, int32_t z, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                     smem_u32(dst)),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
                 : "memory");
}
// an asynchronous copy of 8 bytes (cp_async4 and cp_async16 have the others)
__device__ __forceinline__ void cp_async8(void* smem_dst, const void* gsrc) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(smem_dst)), "l"(gsrc) : "memory");
}
// 16 columns of the warp's 32 lanes
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}

// ---- the kernel

struct alignas(16) TokensSmem {
    TokenLists lists;
    float exchange[16][128];  // the sums of a tile, [slot][row]
    uint64_t full[kMostStages], empty[kMostStages], sums_full[2], sums_free[2], done;
    uint32_t tmem, written;  // written: tiles of up whose silu(g) * u is on its way to the workspace
    int abort;
};
constexpr uint32_t kStageScales = 4 * 512;  // a stage's scale bytes: two atoms (8 bits: one) of each operand
// a stage: the weights' tile, the tokens' columns, the scales of both
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(smem_u32(bar)), "r"(parity)
                 : "memory");
    return ok != 0;
}
// A wait of the block has run out: its other waits end too, and the caller is told.
__device__ __forceinline__ void give_up(volatile int* abort, int32_t* status) {
    *abort = 1;
    if (status) atomicCAS(status, 0, (int32_t)CIERA_ERR_TIMEOUT);
}
// All blocks have added to a counter.  false: the bounded wait ran out, or another of the block's has, or a call before this one was given
// up and the workspace has not been zeros since.
__device__ __forceinline__ bool wait_for_all(const uint32_t* counter, uint32_t blocks, volatile int* abort, int32_t* status) {
    const auto there = [&]() {
        uint32_t seen;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
        if (seen >= kSpoiled) give_up(abort, status);
        return seen >= blocks && seen < kSpoiled;
    };
    return poll(kMaxPolls, there, [&]() { return *abort != 0; }, [&]() { give_up(abort, status); });
}
__device__ __forceinline__ void fence_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// The tiles of a block in both parts, in order: all roles walk them alike.
template <int BITS>
struct TokenWalk {
    const TokensArgs& a;
    const TokenLists& l;
    uint32_t up_tiles, down_tiles, at;
    bool up = true;
    uint32_t group = 0, tile = 0, stages = 0;

    __device__ TokenWalk(const TokensArgs& a_, const TokenLists& l_) : a(a_), l(l_), up_tiles(a_.d_ff / 64), down_tiles(a_.d_model / 128), at(blockIdx.x) {}
    __device__ bool next() {  // false behind the last tile
        if (up) {
            if (at < l.groups * up_tiles) {
                group = at / up_tiles;
                tile = at - group * up_tiles;
                stages = (a.d_model * BITS / 8 + 127) / 128;
                at += gridDim.x;
                return true;
            }
            up = false;
            at = blockIdx.x;
        }
        if (at >= l.groups * down_tiles) return false;
        group = at / down_tiles;
        tile = at - group * down_tiles;
        stages = (a.d_ff * BITS / 8 + 127) / 128;
        at += gridDim.x;
        return true;
    }
    __device__ uint32_t packed() const { return l.group[group]; }
};

// The end of a call (ciera_tokens_end.hpp).  (The router writes its choice and weights while this kernel runs, so they are not read as what
// nobody writes.)
template <int DT>
struct TokensEnd {
    const TokensArgs& a;
    TokensSmem& sm;
    value_t<DT>* out;
    uint32_t tmem;
    bool frees;  // the warp that has allocated tensor memory

    __device__ __forceinline__ void join() {
        __syncthreads();
        if (frees) {
            tensor_fence_after();
            tmem_free_one(tmem, kTokenTmem);
        }
    }
    __device__ __forceinline__ void spoil() {
        if (threadIdx.x == 0) atomicOr(a.counters, kSpoiled);
    }
    __device__ __forceinline__ bool all_done() {
        volatile int* abort = &sm.abort;
        if (threadIdx.x == 0 && !*abort) wait_for_all(a.counters + 2, gridDim.x, abort, a.status);
        __syncthreads();
        return !*abort;
    }
    __device__ __forceinline__ void ticket() {
        if (threadIdx.x == 0) {
            __threadfence();
            if (atomicAdd(a.counters + 3, 1u) == gridDim.x - 1) {
                __threadfence();
                for (int i = 0; i < 4; ++i) a.counters[i] = 0;
            }
        }
    }
    __device__ __forceinline__ void clear() {
        for (uint32_t i = blockIdx.x * kTokenThreads + threadIdx.x; i < sm.lists.groups; i += gridDim.x * kTokenThreads) a.counters[64 + i] = 0;
    }
    // a token's rows, in the order of its choices
    __device__ __forceinline__ void sum() {
        const uint32_t quads = a.d_model / 4;
        value_t<DT>* __restrict__ to_all = out;  // (it may be x, which nobody reads any more; without this 64 tokens 75.6 us, 73.8 so)
        for (uint32_t i = blockIdx.x * kTokenThreads + threadIdx.x; i < a.n_tokens * quads; i += gridDim.x * kTokenThreads) {
            const uint32_t token = i / quads, c = (i - token * quads) * 4;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (uint32_t j0 = 0; j0 < a.top_k; j0 += 8) {
                float4 r[8];
                float wt[8];
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    const uint32_t place = j0 + j < a.top_k ? sm.lists.place[token * a.top_k + j0 + j] : 0xffffu;
                    r[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                    wt[j] = 0.f;
                    if (place != 0xffffu) {
                        r[j] = __ldcg(reinterpret_cast<const float4*>(a.rows + (uint64_t)place * a.d_model + c));
                        wt[j] = a.weights[token * a.top_k + j0 + j];
                    }
                }
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    v[0] = fmaf(wt[j], r[j].x, v[0]);
                    v[1] = fmaf(wt[j], r[j].y, v[1]);
                    v[2] = fmaf(wt[j], r[j].z, v[2]);
                    v[3] = fmaf(wt[j], r[j].w, v[3]);
                }
            }
            value_t<DT>* to = to_all + token * a.out_stride + c;
            if (a.out_wide) {
                store_values<DT, 4>(to, v);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) to[j] = ValueOf<DT>::put(v[j]);
            }
        }
    }
};

template <int DT, int BITS>
__global__ void __launch_bounds__(kTokenThreads, 1)
    tokens_kernel(const TokensArgs a, const __grid_constant__ CUtensorMap w1_map, const __grid_constant__ CUtensorMap w2_map,
                  const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap hidden_map, const value_t<DT>* x,
                  value_t<DT>* out /* may be x */) {
    constexpr uint32_t P = kParts<BITS, DT>;
    constexpr uint32_t kAtoms = BITS == 8 ? 1 : 2;        // of a stage and operand
    extern __shared__ uint8_t tokens_smem[];
    uint8_t* ring = tokens_smem + (-smem_u32(tokens_smem) & 1023u);
    TokensSmem& sm = *reinterpret_cast<TokensSmem*>(ring + a.stages * a.stage_bytes);
    const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, (int)(threadIdx.x >> 5), 0);
    const uint32_t columns_bytes = a.stage_bytes - kTileBytes - kStageScales;
    if (threadIdx.x == 0) {
        prefetch_map(&w1_map);
        prefetch_map(&w2_map);
        prefetch_map(&x_map);
        prefetch_map(&hidden_map);
        for (uint32_t s = 0; s < a.stages; ++s) {
            mbar_init(&sm.full[s], 4);  // the weights' copy, their scales, the columns' copy, theirs
            mbar_init(&sm.empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.sums_full[i], 1);
            mbar_init(&sm.sums_free[i], 4);
        }
        mbar_init(&sm.done, 1);
        sm.abort = 0;
        sm.written = 0;
        mbar_fence_init();
    }
    const uint32_t tid = threadIdx.x & 127;  // of the last four warps, which compute
    const auto all_four = []() { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    const auto done_with = [&](uint32_t* counter) {
        all_four();
        if (tid == 0) {
            __threadfence();
            atomicAdd(counter, 1u);
        }
    };
    if (warp == 2) {
        tmem_alloc_one(&sm.tmem, kTokenTmem);
        tensor_fence_before();
    } else if (warp >= 8) {
        // Before the router has ended: it lets this kernel begin when all that came before it has, the call before this one and whatever
        // wrote x (ciera_route.cuh).
        const uint32_t kbs = a.d_model / 128;
        for (uint32_t u = blockIdx.x * 4 + (warp & 3); u < a.n_tokens * kbs; u += gridDim.x * 4) make_parts<DT, BITS>(a, x, u / kbs, u % kbs, lane);
        done_with(a.counters);
    }
    pdl_wait();
    make_lists(sm.lists, *reinterpret_cast<ListScratch*>(ring), a, kGroupSlots<BITS, DT>);
    tensor_fence_after();
    fence_async_all();  // (what the lists were made in becomes the ring)
    __syncthreads();
    const uint32_t tmem = sm.tmem, blocks = gridDim.x;
    volatile int* abort = &sm.abort;
    TokenWalk<BITS> w(a, sm.lists);
    const auto stage = [&](uint32_t s) { return ring + s * a.stage_bytes; };
    const auto scales_of = [&](uint32_t s) { return ring + s * a.stage_bytes + kTileBytes + columns_bytes; };  // the weights', then the columns'

    if (warp == 0) {
        // copies of weights; they wait for nobody but the tensor cores
        uint32_t it = 0, s = 0, odd = 1;
        bool ok = true;
        while (ok && w.next()) {
            const int32_t e = (int32_t)group_expert(w.packed());
            for (uint32_t k = 0; k < w.stages; ++k, ++it) {
                if (!mbar_wait_soon(&sm.empty[s], odd, abort, a.status)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    mbar_arrive_expect_tx(&sm.full[s], kTileBytes);
                    const int32_t k0 = (int32_t)(k * 128);
                    if (w.up) {
                        map_load3_one(stage(s), &w1_map, k0, (int32_t)(w.tile * 64), e, &sm.full[s]);
                        map_load3_one(stage(s) + kTileBytes / 2, &w1_map, k0, (int32_t)(a.d_ff + w.tile * 64), e, &sm.full[s]);
                    } else {
                        map_load3_one(stage(s), &w2_map, k0, (int32_t)(w.tile * 128), e, &sm.full[s]);
                        map_load3_one(stage(s) + kTileBytes / 2, &w2_map, k0, (int32_t)(w.tile * 128 + 64), e, &sm.full[s]);
                    }
                }
                __syncwarp();
                if (++s == a.stages) s = 0, odd ^= 1;
            }
        }
        if (!ok && lane == 0)  // given up: the copies in flight end before the block does
            for (uint32_t i = it < a.stages ? 0 : it - a.stages; i < it; ++i) {
                int none = 0;
                mbar_wait(&sm.full[i % a.stages], (i / a.stages) & 1, &none, a.status, 1024);
            }
        __syncwarp();
    } else if (warp == 1) {
        // the weights' scales.  8 bits: a byte for 64 or 128 rows, all over an atom's line; 4 bits: the gate's and up's halves of lines
        uint32_t s = 0, odd = 1, back = 0, behind = 0;
        bool ok = true;
        const auto report = [&]() {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.full[back]);
            if (++back == a.stages) back = 0;
            --behind;
        };
        while (ok && w.next()) {
            const Matrices& m = w.up ? a.w1 : a.w2;
            const uint32_t lo = w.up ? w.tile * 64 : w.tile * 128, hi = w.up ? a.d_ff + lo : lo + 64;
            const uint8_t* from = m.scales + group_expert(w.packed()) * m.scales_matrix_stride;
            const uint8_t* a_line = from + (uint64_t)(lo >> 7) * m.scales_stride;
            const uint8_t* b_line = from + (uint64_t)(hi >> 7) * m.scales_stride;
            const uint32_t atoms = (w.up ? a.d_model : a.d_ff) / 128;
            uint32_t a_bytes = 0, b_bytes = 0;  // lane i: of stage k / 32 * 32 + i
            for (uint32_t k = 0; k < w.stages; ++k) {
                if (BITS == 8 && (k & 31) == 0) {
                    if (k + lane < atoms) a_bytes = __ldg(a_line + k + lane), b_bytes = __ldg(b_line + k + lane);
                }
                if (!mbar_wait_soon(&sm.empty[s], odd, abort, a.status)) {
                    ok = false;
                    break;
                }
                uint8_t* to = scales_of(s) + lane * 16;
                if constexpr (BITS == 8) {
                    const uint32_t va = __shfl_sync(~0u, a_bytes, k & 31) * 0x01010101u, vb = __shfl_sync(~0u, b_bytes, k & 31) * 0x01010101u;
                    *reinterpret_cast<uint4*>(to) = make_uint4(va, va, vb, vb);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < kAtoms; ++i)
                        if (k * kAtoms + i < atoms) {
                            const uint64_t off = (uint64_t)(k * kAtoms + i) * kAtomBytes + lane * 16;
                            cp_async8(to + i * 512, a_line + off + (lo & 64 ? 8 : 0));
                            cp_async8(to + i * 512 + 8, b_line + off + (hi & 64 ? 8 : 0));
                        }
                    cp_async_commit();
                }
                ++behind;
                if (++s == a.stages) s = 0, odd ^= 1;
                if (BITS == 8) {
                    report();
                } else if (behind > kBehind) {
                    cp_async_wait<kBehind>();
                    report();
                }
            }
        }
        cp_async_wait<0>();
        while (behind) report();
    } else if (warp == 2) {
        uint32_t it = 0, s = 0, odd = 0, tile = 0;
        bool ok = true;
        const uint32_t stage_units = a.stage_bytes / 16;
        const uint64_t da0 = operand_descriptor(ring), db0 = operand_descriptor(ring + kTileBytes), ds0 = scales_descriptor(scales_of(0));
        while (ok && w.next()) {
            const uint32_t which = tile & 1;
            if (tile >= 2 && !mbar_wait_soon(&sm.sums_free[which], ((tile >> 1) - 1) & 1, abort, a.status)) break;
            tensor_fence_after();
            const uint32_t n = (group_slots(w.packed()) * P + 15) / 16 * 16, d = tmem + which * kSumColumns;
            const uint32_t instruction = BITS == 8 ? mx_instruction(128, n, 0) : mx4_instruction(128, n);
            for (uint32_t k = 0; k < w.stages; ++k, ++it) {
                if (!mbar_wait_soon(&sm.full[s], odd, abort, a.status)) {
                    ok = false;
                    break;
                }
                tensor_fence_after();
                const uint32_t sc = tmem + kTokenScalesAt + (it % kScaleBuffers) * (8 * kAtoms);
                const uint32_t left = w.up ? a.d_model - k * 128 * kAtoms : a.d_ff - k * 128 * kAtoms;  // of the contraction
                if (elect_one()) {
                    const uint64_t da = da0 + s * stage_units, db = db0 + s * stage_units, ds = ds0 + s * stage_units;
#pragma unroll
                    for (uint32_t i = 0; i < 2 * kAtoms; ++i) tmem_copy_scales_one(sc + 4 * i, ds + 32 * i);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (BITS == 8) {
                            tensor_mma_one<8>(d, da + 2 * i, db + 2 * i, instruction + i * mx_byte(1), sc, sc + 4, k > 0 || i > 0);
                        } else {
                            if (i < 2 || left > 128)
                                tensor_mma_one<4>(d, da + 2 * i, db + 2 * i, instruction + (i & 1) * mx_byte(2), sc + 4 * (i >> 1), sc + 8 + 4 * (i >> 1),
                                                  k > 0 || i > 0);
                        }
                    }
                    tensor_commit_one(&sm.empty[s]);
                    if (k + 1 == w.stages) tensor_commit_one(&sm.sums_full[which]);
                }
                __syncwarp();
                if (++s == a.stages) s = 0, odd ^= 1;
            }
            ++tile;
        }
        // nothing that this warp started is in flight when the tensor memory is given back
        if (elect_one()) tensor_commit_one(&sm.done);
        int none = 0;
        mbar_wait_soon(&sm.done, 0, &none, a.status);
        __syncwarp();
    } else if (warp == 3) {
        // tells all blocks of the tiles of up that are written, so that the warps that write them need not wait until they are (128 experts
        // of 256 x 1920 of 34 tokens: 50 us so, 64 by the writing warps)
        if (lane == 0) {
            uint32_t told = 0, there = 0;
            const auto next = [&]() {
                if (!w.next() || !w.up) return false;
                if (there > told) return true;
                const auto written = [&]() {
                    asm volatile("ld.acquire.cta.shared.u32 %0, [%1];" : "=r"(there) : "r"(smem_u32(&sm.written)) : "memory");
                    if (there > told) return true;
                    __nanosleep(32);
                    return false;
                };
                if (!poll(kMaxReportPolls, written, [&]() { return *abort != 0; }, [&]() { give_up(abort, a.status); })) return false;
                __threadfence();
                return true;
            };
            tell(next, [&]() { atomicAdd(a.counters + 64 + w.group, 1u), ++told; }, []() { __threadfence(); }, [&]() { if (told) atomicAdd(a.counters + 1, told); });
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 8) {
        // copies of the tokens' columns and their scale words, behind the blocks that make them; every fourth stage.  (By one warp
        // 64 tokens took 107 us.)
        uint32_t it = 0, s = 0, odd = 1, last = 0;  // last: the warp's stage whose words are on their way
        bool ok, some = false;
        ok = wait_for_all(a.counters, blocks, abort, a.status);
        fence_async_all();  // (written by threads, read by copies)
        const auto report = [&]() {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.full[last]);
            some = false;
        };
        bool all_up = false;  // of all groups
        while (ok && w.next()) {
            if (!w.up && !all_up && takes_part(it, w.stages, warp & 3, kColumnWarps)) {
                uint32_t tiles, whole;
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(tiles) : "l"(a.counters + 64 + w.group) : "memory");
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(whole) : "l"(a.counters + 1) : "memory");
                all_up = __all_sync(~0u, whole >= sm.lists.groups * w.up_tiles);
                if (!all_up && !__all_sync(~0u, tiles >= w.up_tiles)) {
                    if (some) {  // (a tile of up may be waiting for it)
                        cp_async_wait<0>();
                        report();
                    }
                    ok = wait_for_all(a.counters + 64 + w.group, w.up_tiles, abort, a.status);
                    if (!ok) break;
                }
                fence_async_all();
            }
            const uint32_t packed = w.packed(), first = group_first(packed), slots = group_slots(packed);
            const uint32_t atoms = (w.up ? a.d_model : a.d_ff) / 128, rows = a.n_tokens * (w.up ? 1 : a.top_k) * P;
            const uint32_t boxes = (slots * P + 15) / 16, there = min(boxes * 16, rows - (w.up ? 0 : first * P));
            const uint32_t* words = w.up ? a.x_scales : a.hidden_scales;
            uint32_t row[4];  // of the lane's columns lane + 32 * j; none: rows
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t n = j * 32 + lane, slot = n / P;
                row[j] = rows;
                if (w.up) {
                    if (slot < slots) row[j] = sm.lists.token[first + slot] * P + n - slot * P;
                } else if (n < there) {
                    row[j] = first * P + n;
                }
            }
            for (uint32_t k = 0; k < w.stages; ++k, ++it) {
                const uint32_t s_now = s, odd_now = odd;
                if (++s == a.stages) s = 0, odd ^= 1;
                if ((it & (kColumnWarps - 1)) != (uint32_t)(warp & 3)) continue;
                if (some && !__all_sync(~0u, mbar_test(&sm.empty[s_now], odd_now))) {  // no room yet
                    cp_async_wait<0>();
                    report();
                }
                if (!mbar_wait_soon(&sm.empty[s_now], odd_now, abort, a.status)) {
                    ok = false;
                    break;
                }
                // up: a token's parts at a time; down: they lie one behind the other
                if (elect_one()) {
                    uint8_t* to = stage(s_now) + kTileBytes;
                    if (w.up) {
                        mbar_arrive_expect_tx(&sm.full[s_now], slots * P * 128);
                        for (uint32_t i = 0; i < slots; ++i)
                            map_load3_one(to + i * P * 128, &x_map, (int32_t)(k * 128), (int32_t)(sm.lists.token[first + i] * P), 0, &sm.full[s_now]);
                    } else {
                        mbar_arrive_expect_tx(&sm.full[s_now], boxes * 2048);
                        for (uint32_t i = 0; i < boxes; ++i)
                            map_load3_one(to + i * 2048, &hidden_map, (int32_t)(k * 128), (int32_t)(first * P + i * 16), 0, &sm.full[s_now]);
                    }
                }
                __syncwarp();
                uint8_t* to = scales_of(s_now) + kAtoms * 512 + lane * 16;
#pragma unroll
                for (uint32_t i = 0; i < kAtoms; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        if (row[j] < rows && k * kAtoms + i < atoms) cp_async4(to + i * 512 + j * 4, words + (uint64_t)(k * kAtoms + i) * rows + row[j]);
                cp_async_commit();
                if (some) {
                    cp_async_wait<1>();
                    report();
                }
                last = s_now;
                some = true;
            }
        }
        cp_async_wait<0>();
        if (some) report();
        __syncwarp();
    } else if (warp >= 8) {
        // what the tensor cores have finished
        const uint32_t quarter = warp & 3;
        // (they go on or give up together)
        const auto all_agree = [](bool ok) {
            uint32_t r;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(r)
                         : "r"((uint32_t)ok)
                         : "memory");
            return r != 0;
        };
        uint32_t tile = 0;
        bool ok = true;
        while (w.next()) {
            const uint32_t which = tile & 1, packed = w.packed(), slots = group_slots(packed), first = group_first(packed);
            ok = all_agree(mbar_wait_soon(&sm.sums_full[which], (tile >> 1) & 1, abort, a.status, kMaxBarrierPolls + w.stages));
            if (!ok) break;
            tensor_fence_after();
            const uint32_t from = tmem + (quarter << 21) + which * kSumColumns;
            constexpr uint32_t kEach = 16 / P;  // slots of 16 columns
            for (uint32_t slot = 0; slot < slots; slot += kEach) {
                uint32_t r[16];
                tmem_load16(from + slot * P, r);
                tmem_wait_load();
#pragma unroll
                for (uint32_t e = 0; e < kEach; ++e) {
                    if (slot + e >= slots) break;
                    float v = __uint_as_float(r[e * P + P - 1]);  // small ones first
#pragma unroll
                    for (int p = (int)P - 2; p >= 0; --p) v += __uint_as_float(r[e * P + p]);
                    if (w.up) sm.exchange[slot + e][quarter * 32 + lane] = v;
                    else a.rows[(uint64_t)(first + slot + e) * a.d_model + w.tile * 128 + quarter * 32 + lane] = v;
                }
            }
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.sums_free[which]);
            if (w.up) {
                all_four();
                // a warp has 32 columns of the middle, for every other slot
                for (uint32_t slot = quarter >> 1; slot < slots; slot += 2) {
                    const float gate = sm.exchange[slot][(quarter & 1) * 32 + lane], up = sm.exchange[slot][64 + (quarter & 1) * 32 + lane];
                    float v = swiglu32(gate, up);
                    if (gate < kLowestGate) v = (float)((double)gate / (1.0 + exp(-(double)gate)) * (double)up);
                    put_hidden<DT, BITS>(a, v, first + slot, w.tile * 64 + (quarter & 1) * 32, lane);
                }
                all_four();
                if (tid == 0) asm volatile("st.release.cta.shared.u32 [%0], %1;" ::"r"(smem_u32(&sm.written)), "r"(tile + 1) : "memory");
            }
            ++tile;
        }
        if (ok) done_with(a.counters + 2);
    }
    TokensEnd<DT> end{a, sm, out, tmem, warp == 2};
    end_call(end);
}

struct TokensRoom {  // offsets of the workspace's parts
    uint64_t x_parts, x_scales, hidden, hidden_scales, rows, all;
};
// `parts`: ten of 4 bits suffice for every type and format (five of 8 bits take as much room)
static TokensRoom tokens_room(uint64_t tokens, uint64_t top_k, uint64_t d, uint64_t f, uint64_t bits, uint64_t parts) {
    const uint64_t slots = tokens * top_k;
    const auto up = [](uint64_t v) { return (v + 255) / 256 * 256; };
    TokensRoom r;
    r.x_parts = kTokenHead;
    r.x_scales = r.x_parts + up(tokens * parts * d * bits / 8);
    r.hidden = r.x_scales + up(tokens * parts * d / 32);
    r.hidden_scales = r.hidden + up(slots * parts * f * bits / 8);
    r.rows = r.hidden_scales + up(slots * parts * f / 32);
    r.all = r.rows + up(slots * d * 4);
    return r;
}

template <int DT, int BITS>
static cudaError_t launch_tokens(TokensArgs a, const ciera_expert_tokens_args* p, int dev, uint32_t sms, cudaStream_t s) {
    static std::atomic<uint64_t> allowed{0};  // devices on which this instance may have its shared memory
    constexpr uint32_t P = kParts<BITS, DT>, kMost = 227 * 1024 - 1024 - sizeof(TokensSmem);
    // (the lists are made where the ring will be, and stages' scales are reported while there is still room for more)
    static_assert(kMost - (kTileBytes + kMaxColumns * 128 + kStageScales) >= sizeof(ListScratch) &&
                      kMostStages * (kTileBytes + 2048 + kStageScales) >= sizeof(ListScratch) &&
                      kMost / (kTileBytes + kMaxColumns * 128 + kStageScales) > kBehind,
                  "too short a ring");
    const uint64_t slots = (uint64_t)a.n_tokens * a.top_k, d = a.d_model, f = a.d_ff;
    const TokensRoom room = tokens_room(a.n_tokens, a.top_k, d, f, BITS, P);
    uint8_t* const base = (uint8_t*)p->workspace;
    a.x_parts = base + room.x_parts;
    a.x_scales = (uint32_t*)(base + room.x_scales);
    a.hidden = base + room.hidden;
    a.hidden_scales = (uint32_t*)(base + room.hidden_scales);
    a.rows = (float*)(base + room.rows);
    // columns of a group at most (no token is there twice), and the stages that there is room for
    const uint32_t group = a.n_tokens < kGroupSlots<BITS, DT> ? a.n_tokens : kGroupSlots<BITS, DT>;
    a.stage_bytes = kTileBytes + (group * P + 15) / 16 * 2048 + kStageScales;
    a.stages = kMost / a.stage_bytes < (uint32_t)kMostStages ? kMost / a.stage_bytes : (uint32_t)kMostStages;
    CUtensorMap w1, w2, xm, hm;
    if (!operand_map(&w1, p->w1, d * BITS / 8, 2 * f, a.n_experts, p->w1_stride, p->w1_matrix_stride, 64) ||
        !operand_map(&w2, p->w2, f * BITS / 8, d, a.n_experts, p->w2_stride, p->w2_matrix_stride, 64) ||
        !operand_map(&xm, a.x_parts, d * BITS / 8, (uint64_t)a.n_tokens * P, 1, d * BITS / 8, 0, P) ||
        !operand_map(&hm, a.hidden, f * BITS / 8, slots * P, 1, f * BITS / 8, 0, 16))
        return cudaErrorInvalidValue;
    auto kernel = tokens_kernel<DT, BITS>;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    // no more blocks than have work in one of the parts
    const uint64_t up = slots * (f / 64), down = slots * (d / 128), work = up > down ? up : down;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)(work < sms ? work : sms));
    cfg.blockDim = dim3(kTokenThreads);
    cfg.dynamicSmemBytes = 1024 + a.stages * a.stage_bytes + sizeof(TokensSmem);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, w1, w2, xm, hm, (const value_t<DT>*)p->x, (value_t<DT>*)p->out);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace ciera

using namespace ciera;

extern "C" size_t ciera_expert_tokens_workspace_bytes(uint32_t n_tokens, uint32_t top_k, uint32_t d_model, uint32_t d_ff) {
    return tokens_room(n_tokens, top_k, d_model, d_ff, 4, 10).all;
}

extern "C" int ciera_expert_tokens(const ciera_expert_tokens_args* p, void* stream) {
    if (!p || p->n_tokens > CIERA_EXPERT_TOKENS_MAX) return CIERA_ERR_INVALID_ARG;
    if (p->dtype != CIERA_BF16 && p->dtype != CIERA_FP32 && p->dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if (p->format != CIERA_WEIGHTS_FP8 && p->format != CIERA_WEIGHTS_FP4) return CIERA_ERR_INVALID_ARG;
    const uint64_t d = p->d_model, f = p->d_ff, t = p->n_tokens, E = p->route.n_experts;
    if (d < 128 || f < 128 || (d & 127) || (f & 127) || d > 65536 || f > 65536) return CIERA_ERR_INVALID_ARG;
    if (t && (!p->x || !p->out || !p->w1 || !p->w1_scales || !p->w2 || !p->w2_scales || !p->workspace)) return CIERA_ERR_INVALID_ARG;
    if (t > 1 && (p->x_stride < d || p->out_stride < d)) return CIERA_ERR_INVALID_ARG;
    const bool four = p->format == CIERA_WEIGHTS_FP4;
    // bytes of a row of codes and of a line of scales, and how many lines (strides of single lines count for nothing)
    const auto weights = [&](const void* q, uint64_t stride, uint64_t matrix_stride, const void* scales, uint64_t scales_stride,
                             uint64_t scales_matrix_stride, uint64_t rows, uint64_t cols) {
        const uint64_t line = four ? cols / 2 : cols, scale_line = four ? cols / 128 * kAtomBytes : cols / 128;
        if (stride < line || (rows > 128 && scales_stride < scale_line)) return (int)CIERA_ERR_INVALID_ARG;
        if (!aligned_to(q, 16) || (stride & 15) || (E > 1 && (matrix_stride & 15))) return (int)CIERA_ERR_MISALIGNED;
        if (four && (!aligned_to(scales, 16) || (rows > 128 && (scales_stride & 511)) || (E > 1 && (scales_matrix_stride & 15)))) return (int)CIERA_ERR_MISALIGNED;
        if (stride >= 1ull << 40 || (E > 1 && matrix_stride >= 1ull << 40)) return (int)CIERA_ERR_UNSUPPORTED;
        return (int)CIERA_OK;
    };
    if (t) {
        int rc = weights(p->w1, p->w1_stride, p->w1_matrix_stride, p->w1_scales, p->w1_scales_stride, p->w1_scales_matrix_stride, 2 * f, d);
        if (!rc) rc = weights(p->w2, p->w2_stride, p->w2_matrix_stride, p->w2_scales, p->w2_scales_stride, p->w2_scales_matrix_stride, d, f);
        if (rc) return rc;
        if (!aligned_to(p->x, dtype_bytes(p->dtype)) || !aligned_to(p->out, dtype_bytes(p->dtype)) || !aligned_to(p->workspace, 16) ||
            !aligned_to(p->status, 4))
            return CIERA_ERR_MISALIGNED;
        if (p->workspace_bytes < ciera_expert_tokens_workspace_bytes(p->n_tokens, p->route.top_k, p->d_model, p->d_ff)) return CIERA_ERR_CAPACITY;
    }
    int rc = check_route(&p->route, p->logits_dtype, p->logits, t, p->logits_stride, p->bias, p->experts, p->weights);
    if (rc || !t) return rc;
    int dev = 0, sms = 0;
    rc = device_and_sms(&dev, &sms);
    if (rc) return rc;
    if (!encode_tiled()) return record_cuda_error(cudaErrorNotSupported);
    rc = ciera_route(&p->route, p->logits_dtype, p->logits, t, p->logits_stride, p->bias, p->experts, p->weights, stream);
    if (rc) return rc;
    const uint64_t v = dtype_bytes(p->dtype);
    TokensArgs a = {};
    a.w1 = Matrices{p->w1_scales, p->w1_scales_stride, p->w1_scales_matrix_stride};
    a.w2 = Matrices{p->w2_scales, p->w2_scales_stride, p->w2_scales_matrix_stride};
    a.experts = p->experts;
    a.weights = p->weights;
    a.x_stride = p->x_stride;
    a.out_stride = p->out_stride;
    a.counters = (uint32_t*)p->workspace;
    a.status = p->status;
    a.n_tokens = (uint32_t)t;
    a.top_k = p->route.top_k;
    a.n_experts = p->route.n_experts;
    a.d_model = (uint32_t)d;
    a.d_ff = (uint32_t)f;
    a.x_wide = !(((uint64_t)p->x | (t > 1 ? p->x_stride * v : 0)) & (4 * v - 1));
    a.out_wide = !(((uint64_t)p->out | (t > 1 ? p->out_stride * v : 0)) & (4 * v - 1));
    cudaError_t e = cudaSuccess;
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        e = four ? launch_tokens<DT, 4>(a, p, dev, (uint32_t)sms, (cudaStream_t)stream) : launch_tokens<DT, 8>(a, p, dev, (uint32_t)sms, (cudaStream_t)stream);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    return CIERA_OK;
}
