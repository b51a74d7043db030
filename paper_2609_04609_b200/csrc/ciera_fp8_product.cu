// Products of e4m3 operands with a power of two for each block of 128 values of the contraction.
//
// out = sum over blocks b of 2^(sa + sb) * a_b * b_b^T.  The tensor cores take a power of two for each row and 32 values
// (kind::mxf8f6f4), so a block's scale is handed to them four times over and the sum over all blocks stays in tensor memory in
// fp32: no result passes through registers before the last block.
//
// Persistent pairs of blocks of threads (a cluster on two SMs) take tiles of 256 columns x 256 (or 128) rows of out.  b's rows
// are the tensor cores' first operand, 128 to a block, a's rows the second, half of them to a block: a block then writes and reads
// 32 KB of its shared memory for 128 values of the contraction, in the 512 cycles that the products take, where a block on
// 128 x 256 of its own would have to move 48 KB.  b's rows in front, since segments of a's end at any multiple of 128: a
// tile's second half is left out where its segment has no rows for it, in both blocks.  (Such a tile costs three quarters of
// a whole one.)
//   warp 0      copies tiles of a and b (128 values of the contraction) into a ring of stages by tensor maps
//   warp 1      of the first block: starts a stage's four products; before every fourth stage of a tile it copies the scales
//               of four into tensor memory
//   warps 2, 3  read the scale bytes of four stages at a time, each in turn, and lay them out as the tensor cores want them:
//               row r's four bytes in word r / 32 of line r % 32.  (A stage at a time, with its byte four times over, cost a
//               third of the time of the whole: 8192^3 took 606 us, 399 without any scales.)
//   warps 4-7   read finished sums (a lane is a column of out) and write them
// Two sums are in flight, so a tile's products run while the one before is written.  Tensor memory has 512 columns: the two sums
// share 64 of them, which are the first that are read (the next tile's products wait for them alone), and 64 hold the scales of
// four groups of stages.
//
// What a block does for the other is ordered in the cluster's scope: scales by a release and an acquire of shared memory, sums that
// have been read by the tensor fences; and a block leaves when every arrival on its barriers has come.  (Orders of the block's
// own scope and no wait at the end: one token on 8 experts 11.9 us, 13.5 so; large products the same.)
//
// Measured: 8192^3 406 us, 2710 TFLOP/s (a first form with one block on 128 x 256 and a byte of scales four times over 504);
// 32768 rows of 64 experts, 2048 x 2048, 142 us forward and 227 us for the weights' gradient, 1074 MB of fp32 results at 83% of the
// copy rate; one token on 8 experts 13.5 us, of which DRAM needs 5.  A copy of this that starts all products and waits for nothing
// takes 93 us forward; the rest is the change from one tile's sum to the next, copies that come late, and writing.  Tried
// and slower: tiles brought into L2 ahead of their copies (forward 144 -> 149 to 156 us, 8192^3 394 -> 413 to 456); two tiles of 128
// rows to a pair as often as one of 256 (144 -> 150 us).
#include <cuda.h>

#include <type_traits>

#include "ciera_numeric.cuh"
#include "ciera_tensor.cuh"

namespace ciera {

constexpr int kProductThreads = 256;
constexpr int kStages = 6;
constexpr uint32_t kTileN = 256;  // columns of a pair's tile
constexpr int kGroup = 4;         // stages whose scales go together: a byte each in a word
constexpr int kGroups = 4;        // such groups in shared and in tensor memory
constexpr uint32_t kMaxSegments = 1024;
constexpr uint32_t kShared = 64, kSecondSum = 256 - kShared, kScalesAt = kSecondSum + 256;  // columns of tensor memory

struct ProductArgs {
    uint64_t a_scales_stride, b_scales_stride, b_scales_matrix_stride, out_stride, out_matrix_stride;
    const uint8_t* a_scales;
    const uint8_t* b_scales;
    const int32_t* starts;
    int32_t* status;
    uint32_t m, n, k, n_experts;
    int32_t a_words, b_words;  // scale bytes of rows may be read four at a time
    int32_t b_blocks;
    int32_t wide_out;     // 16-bit columns of out may be written two at a time
    uint32_t tile_m;      // rows of a tile: 256 or 128
};

struct alignas(1024) ProductSmem {
    uint8_t b[kStages][128 * 128];
    uint8_t a[kStages][128 * 128];
    uint32_t b_scales[kGroups][128];
    uint32_t a_scales[kGroups][2][128];
    uint64_t full[kStages], empty[kStages], scales_full[kGroups], scales_empty[kGroups], sums_full[2], sums_free[2], done;
    uint32_t tmem;
    int abort;
    int32_t starts[kMaxSegments + 1];
    uint32_t first_tile[kMaxSegments + 1];  // rows' tiles before each segment
};

static_assert(sizeof(ProductSmem) + 1024 <= 227 * 1024, "more than a block may have");

// The tiles of a pair, in order, and the blocks of the contraction in each.
template <int MODE>
struct Walk {
    const ProductArgs& p;
    const ProductSmem& sm;
    uint32_t n_tiles, m_tiles, all, at;
    uint32_t e = 0, m0 = 0, n0 = 0, m1 = 0, kb0 = 0, kb1 = 0;

    __device__ Walk(const ProductArgs& p_, const ProductSmem& sm_) : p(p_), sm(sm_), at(blockIdx.x >> 1) {
        n_tiles = (p.n + kTileN - 1) / kTileN;
        m_tiles = MODE == CIERA_PRODUCT_ROWS ? sm.first_tile[p.n_experts] : (p.m + p.tile_m - 1) / p.tile_m;
        all = m_tiles * n_tiles * (MODE == CIERA_PRODUCT_CONTRACT ? p.n_experts : 1u);
    }
    __device__ bool next() {  // false behind the last tile
        if (at >= all) return false;
        const uint32_t row = at / n_tiles;
        n0 = (at - row * n_tiles) * kTileN;
        if (MODE == CIERA_PRODUCT_CONTRACT) {
            e = row / m_tiles;
            m0 = (row - e * m_tiles) * p.tile_m;
            m1 = p.m;
            kb0 = (uint32_t)sm.starts[e] / 128;
            kb1 = (uint32_t)sm.starts[e + 1] / 128;
        } else {
            if (MODE == CIERA_PRODUCT_ROWS) {
                while (sm.first_tile[e + 1] <= row) ++e;  // (tiles come in rising order)
                m0 = (uint32_t)sm.starts[e] + (row - sm.first_tile[e]) * p.tile_m;
                m1 = (uint32_t)sm.starts[e + 1];
            } else {
                m0 = row * p.tile_m;
                m1 = p.m;
            }
            kb0 = 0;
            kb1 = (p.k + 127) / 128;
        }
        at += gridDim.x >> 1;
        return true;
    }
    // rows of the tile that the products are made for
    __device__ uint32_t height() const { return m1 - m0 > 128 && p.tile_m == 256 ? 256u : 128u; }
};

// 128 scale bytes of a block, four rows a lane: rows row0 + 4 * lane ...; the bytes of rows from `rows` on do not matter.  words:
// lines start at multiples of four (the rest of a word that holds a row's byte is read with it).  Nothing is done with what
// is read, so that all of a group's loads are on their way together.
__device__ __forceinline__ uint32_t row_scales(const uint8_t* line, uint32_t row0, uint32_t rows, bool words, int lane) {
    const uint32_t r = row0 + 4 * lane;
    uint32_t v = 0x7f7f7f7fu;
    if (words) {
        if (r < rows) v = __ldg(reinterpret_cast<const uint32_t*>(line + r));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i < rows) v = (v & ~(255u << (8 * i))) | (uint32_t)__ldg(line + r + i) << (8 * i);
    }
    return v;
}
// Scale bytes of four blocks, four rows a lane in each, to words of a row's four bytes: row r in word r / 32 of line r % 32.
__device__ __forceinline__ void lay_out_scales(uint32_t* to, const uint32_t (&v)[kGroup], int lane) {
    const uint32_t lo01 = __byte_perm(v[0], v[1], 0x5140), hi01 = __byte_perm(v[0], v[1], 0x7362);
    const uint32_t lo23 = __byte_perm(v[2], v[3], 0x5140), hi23 = __byte_perm(v[2], v[3], 0x7362);
    uint32_t* w = to + (lane & 7) * 16 + (lane >> 3);
    w[0] = __byte_perm(lo01, lo23, 0x5410);
    w[4] = __byte_perm(lo01, lo23, 0x7632);
    w[8] = __byte_perm(hi01, hi23, 0x5410);
    w[12] = __byte_perm(hi01, hi23, 0x7632);
}

// Two sums rounded to a 16-bit type, the first in the low half.
template <int DT>
__device__ __forceinline__ uint32_t pack_two(uint32_t lo, uint32_t hi) {
    const float x = __uint_as_float(lo), y = __uint_as_float(hi);
    if constexpr (DT == CIERA_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}

// Writes 32 columns x 32 rows of out of which the lane has column `col` in r: neighbouring columns are in neighbouring lanes, so
// a row goes out as it is, 16-bit values two at a time: an even lane puts row c's together, its neighbour row c + 1's.
template <int DT>
__device__ __forceinline__ void write_part(const uint32_t (&r)[32], value_t<DT>* out, uint64_t stride, uint32_t row, uint32_t rows,
                                           uint32_t col, uint32_t cols, bool wide, int lane) {
    if constexpr (DT == CIERA_FP32) {
        uint32_t* to = reinterpret_cast<uint32_t*>(out + row * stride + col);
        if (col >= cols) return;
        if (row + 32 <= rows) {
#pragma unroll
            for (int c = 0; c < 32; ++c, to += stride) *to = r[c];
        } else {
#pragma unroll
            for (int c = 0; c < 32; ++c, to += stride)
                if (row + c < rows) *to = r[c];
        }
    } else if (wide) {
        const uint32_t odd = lane & 1;
        uint32_t* to = reinterpret_cast<uint32_t*>(out + (row + odd) * stride + (col - odd));
        const bool some = col - odd < cols;  // (cols is even)
        const bool all = row + 32 <= rows;
#pragma unroll
        for (int c = 0; c < 32; c += 2, to += stride) {
            const uint32_t other = __shfl_xor_sync(~0u, odd ? r[c] : r[c + 1], 1);
            const uint32_t both = odd ? pack_two<DT>(other, r[c + 1]) : pack_two<DT>(r[c], other);
            if (some && (all || row + c + odd < rows)) *to = both;
        }
    } else {
        value_t<DT>* to = out + row * stride + col;
#pragma unroll
        for (int c = 0; c < 32; ++c, to += stride)
            if (col < cols && row + c < rows) *to = ValueOf<DT>::put(__uint_as_float(r[c]));
    }
}

template <int MODE, int DT>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const ProductArgs p, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                   value_t<DT>* __restrict__ out) {
    extern __shared__ uint8_t product_smem[];
    ProductSmem& sm = *reinterpret_cast<ProductSmem*>(product_smem + (-smem_u32(product_smem) & 1023u));
    const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, (int)(threadIdx.x >> 5), 0);
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.empty[s], 1);
        }
        for (int g = 0; g < kGroups; ++g) {
            mbar_init(&sm.scales_full[g], 2);  // (the first block's) a warp of each block
            mbar_init(&sm.scales_empty[g], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.sums_full[i], 1);
            mbar_init(&sm.sums_free[i], 8);  // (the first block's) both blocks' writing warps
        }
        mbar_init(&sm.done, 1);
        sm.abort = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        tmem_alloc(&sm.tmem, 512);
        tensor_fence_before();
    }
    pdl_wait();
    bool bad = false;
    if (MODE != CIERA_PRODUCT_DENSE) {
        const uint32_t most = MODE == CIERA_PRODUCT_CONTRACT ? p.k : p.m;
        for (uint32_t i = threadIdx.x; i <= p.n_experts; i += kProductThreads) {
            const int32_t v = p.starts[i], before = i ? p.starts[i - 1] : 0;
            sm.starts[i] = v;
            bad |= v < before || (v & 127) || (uint32_t)v > most || (i == 0 && v != 0);
        }
    }
    bad = __syncthreads_or(bad);
    if (MODE == CIERA_PRODUCT_ROWS && !bad) {
        if (warp == 0) {
            uint32_t run = 0;
            for (uint32_t e0 = 0; e0 < p.n_experts; e0 += 32) {
                const uint32_t e = e0 + lane;
                const uint32_t v = e < p.n_experts ? ((uint32_t)(sm.starts[e + 1] - sm.starts[e]) + p.tile_m - 1) / p.tile_m : 0;
                uint32_t s = v;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t o = __shfl_up_sync(~0u, s, d);
                    if (lane >= d) s += o;
                }
                if (e < p.n_experts) sm.first_tile[e] = run + s - v;
                run += __shfl_sync(~0u, s, 31);
            }
            if (lane == 0) sm.first_tile[p.n_experts] = run;
        }
    }
    tensor_fence_before();
    cluster_sync();  // barriers, tables and tensor memory of both blocks are there
    tensor_fence_after();
    const uint32_t tmem = sm.tmem;
    if (bad) {  // (in both blocks: they read the same table)
        if (p.status && threadIdx.x == 0 && rank == 0) atomicCAS(p.status, 0, (int32_t)CIERA_ERR_CORRUPT);
        if (warp == 1) tmem_free(tmem, 512);
        return;
    }
    Walk<MODE> w(p, sm);
    volatile int* abort = &sm.abort;
    uint32_t it = 0;  // blocks of the contraction so far

    if (warp == 0) {
        bool ok = true;
        uint32_t s = 0, odd = 1;  // stage, and the parity of its last phase
        while (ok && w.next()) {
            const uint32_t half = w.height() / 2;
            const int32_t m0 = (int32_t)(w.m0 + rank * half), n0 = (int32_t)(w.n0 + rank * 128);
            for (uint32_t kb = w.kb0; kb < w.kb1; ++kb, ++it) {
                if (!mbar_wait_soon(&sm.empty[s], odd, abort, p.status)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx(&sm.full[s], 2 * (128 * 128 + half * 128));
                    const uint32_t full = in_first_block(&sm.full[s]);
                    const int32_t k0 = (int32_t)(kb * 128);
                    map_load3(sm.b[s], &b_map, k0, n0, MODE == CIERA_PRODUCT_ROWS ? (int32_t)w.e : 0, full);
                    map_load3(sm.a[s], &a_map, k0, m0, 0, full);
                    if (half == 128) map_load3(sm.a[s] + 64 * 128, &a_map, k0, m0 + 64, 0, full);
                }
                __syncwarp();
                if (++s == kStages) s = 0, odd ^= 1;
            }
        }
        // No block leaves while an arrival is on its way to one of its barriers: those that nobody else waits for are waited for
        // here, and with them all products that read the stages.
        const uint32_t since = it < kStages ? 0 : it - kStages;
        if (ok) {
            for (uint32_t i = since; i < it; ++i) mbar_wait_soon(&sm.empty[i % kStages], (i / kStages) & 1, abort, p.status);
        } else if (rank == 0 && lane == 0) {  // given up: the copies in flight (they report to the first block) end before the cluster does
            for (uint32_t i = since; i < it; ++i) {
                int none = 0;
                mbar_wait(&sm.full[i % kStages], (i / kStages) & 1, &none, p.status, 1024);
            }
        }
        __syncwarp();
        // (the first block's warp 1 waits for its own; it gives up at most one bound later than this block's warps)
        if (rank == 1) {
            int none = 0;
            mbar_wait_soon(&sm.done, 0, &none, p.status, 3 * kMaxBarrierPolls);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            uint32_t tile = 0, g = 0, g_odd = 0, s = 0, odd = 0;
            bool ok = true;
            const uint64_t db0 = operand_descriptor(sm.b[0]), da0 = operand_descriptor(sm.a[0]);
            while (ok && w.next()) {
                if (w.kb0 == w.kb1) continue;
                if (tile) {  // the columns shared with the sum before have been read
                    if (!mbar_wait_cluster(&sm.sums_free[(tile - 1) & 1], ((tile - 1) >> 1) & 1, abort, p.status)) break;
                    tensor_fence_after();
                }
                const uint32_t first = mx_instruction(256, w.height(), 0), d = tmem + (tile & 1) * kSecondSum;
                uint32_t j = 0;
                for (uint32_t kb = w.kb0; kb < w.kb1; ++kb) {
                    const uint32_t sc = tmem + kScalesAt + 16 * g;
                    if (!mbar_wait_soon(&sm.full[s], odd, abort, p.status) ||
                        (j == 0 && !mbar_wait_cluster(&sm.scales_full[g], g_odd, abort, p.status))) {
                        ok = false;
                        break;
                    }
                    if (j == 0) fence_acquire_shared();
                    tensor_fence_after();
                    const bool last = kb + 1 == w.kb1;
                    if (elect_one()) {
                        if (j == 0) {
                            tmem_copy_scales(sc, scales_descriptor(sm.b_scales[g]));
                            tmem_copy_scales(sc + 8, scales_descriptor(sm.a_scales[g][0]));
                            tmem_copy_scales(sc + 12, scales_descriptor(sm.a_scales[g][1]));
                        }
                        const uint64_t db = db0 + s * (128 * 128 / 16), da = da0 + s * (128 * 128 / 16);
                        const uint32_t instruction = first + j * mx_byte(1);
#pragma unroll
                        for (int i = 0; i < 4; ++i) tensor_mma_mx(d, db + 2 * i, da + 2 * i, instruction, sc, sc + 8, kb > w.kb0 || i > 0);
                        tensor_commit(&sm.empty[s]);
                        if (j == kGroup - 1 || last) tensor_commit(&sm.scales_empty[g]);
                        if (last) tensor_commit(&sm.sums_full[tile & 1]);
                    }
                    __syncwarp();
                    if (++s == kStages) s = 0, odd ^= 1;
                    if (++j == kGroup || last) {
                        j = 0;
                        if (++g == kGroups) g = 0, g_odd ^= 1;
                    }
                }
                ++tile;
            }
            // nothing that this warp started is in flight when the tensor memory is given back
            if (elect_one()) tensor_commit(&sm.done);
            int none = 0;
            mbar_wait_soon(&sm.done, 0, &none, p.status);
        }
        __syncwarp();
    } else if (warp < 4) {
        // this warp's groups are every other one; the next one's bytes are on their way while it waits for room
        uint32_t kb = 0, group = 0;
        bool more = w.next();
        auto settle = [&]() {  // to the next block of the contraction that there is
            while (more && kb >= w.kb1) {
                more = w.next();
                kb = w.kb0;
            }
        };
        auto skip = [&]() {
            if (more) kb = min(kb + kGroup, w.kb1);
            settle();
        };
        uint32_t vb[kGroup], va0[kGroup], va1[kGroup];
        bool some = false;
        auto fetch = [&]() {
            some = more;
            if (!more) return;
            const uint32_t n0 = w.n0 + 128 * rank;
            const uint8_t* block = p.b_scales + (MODE == CIERA_PRODUCT_ROWS ? w.e : 0) * p.b_scales_matrix_stride + (uint64_t)(n0 / 128) * p.b_scales_stride;
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                vb[j] = va0[j] = va1[j] = 127u;
                const uint32_t k = kb + j;
                if (k >= w.kb1) continue;
                if (!p.b_blocks) vb[j] = row_scales(p.b_scales + k * p.b_scales_stride, n0, p.n, p.b_words, lane);
                else if (n0 < p.n) vb[j] = __ldg(block + k);
                va0[j] = row_scales(p.a_scales + k * p.a_scales_stride, w.m0, w.m1, p.a_words, lane);
                va1[j] = row_scales(p.a_scales + k * p.a_scales_stride, w.m0 + 128, w.m1, p.a_words, lane);
            }
            skip();
        };
        kb = w.kb0;
        settle();
        if (warp == 3) {
            skip();
            group = 1;
        }
        fetch();
        bool ok = true;
        while (some) {
            const uint32_t g = group % kGroups;
            if (!mbar_wait_soon(&sm.scales_empty[g], ((group / kGroups) & 1) ^ 1, abort, p.status)) {
                ok = false;
                break;
            }
            if (p.b_blocks) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j) vb[j] *= 0x01010101u;
            }
            lay_out_scales(sm.b_scales[g], vb, lane);
            lay_out_scales(sm.a_scales[g][0], va0, lane);
            lay_out_scales(sm.a_scales[g][1], va1, lane);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(in_first_block(&sm.scales_full[g]));
            group += 2;
            skip();
            fetch();
        }
        // (as in warp 0: the last groups' arrivals)
        for (uint32_t back = 4; ok && back; back -= 2)
            if (group >= back) ok = mbar_wait_soon(&sm.scales_empty[(group - back) % kGroups], ((group - back) / kGroups) & 1, abort, p.status);
        __syncwarp();
    } else {
        const int quarter = warp & 3;
        uint32_t tile = 0;
        while (w.next()) {
            const uint32_t n = w.n0 + rank * 128 + quarter * 32;
            value_t<DT>* o = out + (MODE == CIERA_PRODUCT_CONTRACT ? w.e * p.out_matrix_stride : 0);
            auto write = [&](const uint32_t(&r)[32], uint32_t part) {
                write_part<DT>(r, o, p.out_stride, w.m0 + 32 * part, w.m1, n + lane, p.n, p.wide_out, lane);
            };
            const uint32_t parts = w.height() / 32;
            if (w.kb0 == w.kb1) {  // nothing to add up
                const uint32_t zero[32] = {};
                for (uint32_t i = 0; i < parts; ++i) write(zero, i);
                continue;
            }
            const uint32_t which = tile & 1;
            if (!mbar_wait_soon(&sm.sums_full[which], (tile >> 1) & 1, abort, p.status, kMaxBarrierPolls + (w.kb1 - w.kb0))) break;
            __syncwarp();
            tensor_fence_after();
            const uint32_t from = tmem + ((uint32_t)quarter << 21) + which * kSecondSum;
            // the columns shared with the other sum first: the second's first two parts, the first's last two of eight
            const uint32_t first = which == 0 && parts == 8 ? 6 : 0;
            uint32_t r[2][32];
#pragma unroll
            for (int i = 0; i < 2; ++i) tmem_load32(from + 32 * (first + i), r[i]);
            tmem_wait_load();
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_read(in_first_block(&sm.sums_free[which]));
#pragma unroll
            for (int i = 0; i < 2; ++i) write(r[i], first + i);
            for (uint32_t i = 2; i < parts; ++i) {
                const uint32_t part = first ? i - 2 : i;
                tmem_load32(from + 32 * part, r[0]);
                tmem_wait_load();
                write(r[0], part);
            }
            ++tile;
        }
        __syncwarp();
    }
    tensor_fence_before();
    cluster_sync();  // neither block's memory is in use by the other
    if (warp == 1) {
        tensor_fence_after();
        tmem_free(tmem, 512);
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return f;
}

// Tiles of 128 bytes x `box` rows of [matrices][rows, k] bytes; what lies outside arrives as zero.
static bool operand_map(CUtensorMap* map, const void* p, uint64_t k, uint64_t rows, uint64_t matrices, uint64_t stride,
                        uint64_t matrix_stride, uint32_t box) {
    const uint64_t line = (k + 15) & ~15ull;
    if (rows <= 1) stride = line;  // (never stepped by)
    if (matrices <= 1) matrix_stride = stride;
    const cuuint64_t dims[3] = {k, rows, matrices}, strides[2] = {stride, matrix_stride};
    const cuuint32_t boxes[3] = {128, box, 1}, steps[3] = {1, 1, 1};
    return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(p), dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the current device and its SMs
static int device_and_sms(int* dev, int* n) {
    static std::atomic<int> known[64];
    cudaError_t e = cudaGetDevice(dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (*dev < 64 && (*n = known[*dev].load(std::memory_order_relaxed)) > 0) return CIERA_OK;
    e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, *dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (*dev < 64) known[*dev].store(*n, std::memory_order_relaxed);
    return CIERA_OK;
}

template <int MODE, int DT>
static cudaError_t launch_product(const ProductArgs& a, const CUtensorMap& am, const CUtensorMap& bm, void* out, uint32_t pairs, int dev, cudaStream_t s) {
    static std::atomic<uint64_t> allowed{0};  // devices on which this instance may have its shared memory
    constexpr size_t smem = sizeof(ProductSmem) + 1024;  // (the ring starts at a multiple of 1024)
    auto kernel = product_kernel<MODE, DT>;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * pairs);
    cfg.blockDim = dim3(kProductThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, am, bm, (value_t<DT>*)out);
}

}  // namespace ciera

using namespace ciera;

extern "C" int ciera_fp8_matmul(const ciera_fp8_product* p, void* stream) {
    if (!p) return CIERA_ERR_INVALID_ARG;
    const int mode = p->mode;
    if (mode != CIERA_PRODUCT_DENSE && mode != CIERA_PRODUCT_ROWS && mode != CIERA_PRODUCT_CONTRACT) return CIERA_ERR_INVALID_ARG;
    if (p->out_dtype != CIERA_BF16 && p->out_dtype != CIERA_FP32 && p->out_dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    const bool rows = mode == CIERA_PRODUCT_ROWS, contract = mode == CIERA_PRODUCT_CONTRACT;
    if (p->m < 1 || p->n < 1 || p->k < 1 || p->m > kMaxExtent || p->n > kMaxExtent || p->k > kMaxExtent) return CIERA_ERR_INVALID_ARG;
    if (!p->a || !p->a_scales || !p->b || !p->b_scales || !p->out || (p->b_blocks != 0 && p->b_blocks != 1) ||
        (rows && !p->b_blocks) || (contract && p->b_blocks) || ((rows || contract) != (p->starts != nullptr)) ||
        ((rows || contract) && (p->n_experts < 1 || p->n_experts > kMaxSegments)))
        return CIERA_ERR_INVALID_ARG;
    const uint64_t kb = (p->k + 127) / 128, nb = (p->n + 127) / 128;
    if ((p->m > 1 && p->a_stride < p->k) || (p->n > 1 && p->b_stride < p->k) || (kb > 1 && p->a_scales_stride < p->m) ||
        (p->b_blocks ? nb > 1 && p->b_scales_stride < kb : kb > 1 && p->b_scales_stride < p->n) || (p->m > 1 && p->out_stride < p->n))
        return CIERA_ERR_INVALID_ARG;
    // (strides of single rows and matrices count for nothing)
    const bool several = rows && p->n_experts > 1;
    if (!aligned_to(p->a, 16) || !aligned_to(p->b, 16) || (p->m > 1 && (p->a_stride & 15)) || (p->n > 1 && (p->b_stride & 15)) ||
        (several && (p->b_matrix_stride & 15)) || !aligned_to(p->out, dtype_bytes(p->out_dtype)) || !aligned_to(p->starts, 4) ||
        !aligned_to(p->status, 4))
        return CIERA_ERR_MISALIGNED;
    if ((p->m > 1 && p->a_stride >= 1ull << 40) || (p->n > 1 && p->b_stride >= 1ull << 40) || (several && p->b_matrix_stride >= 1ull << 40))
        return CIERA_ERR_UNSUPPORTED;
    int dev = 0, sms = 0;
    const int rc = device_and_sms(&dev, &sms);
    if (rc) return rc;
    // tiles of 128 rows where those of 256 would leave SMs without work (every segment has at most one more than its rows fill)
    const uint64_t groups = contract ? p->n_experts : 1, n_tiles = (p->n + kTileN - 1) / kTileN, pairs = sms / 2;
    const auto tiles_of = [&](uint64_t h) { return ((p->m + h - 1) / h) * n_tiles * groups; };
    const uint32_t tile_m = tiles_of(256) >= pairs ? 256 : 128;
    const uint64_t tiles = tiles_of(tile_m) + (rows && tile_m == 256 ? p->n_experts * n_tiles : 0);
    if (tiles > 0xffffffffull - 65536) return CIERA_ERR_UNSUPPORTED;
    const uint32_t grid = (uint32_t)(tiles < pairs ? tiles : pairs);
    const bool words_a = aligned_to(p->a_scales, 4) && !(p->a_scales_stride & 3), words_b = aligned_to(p->b_scales, 4) && !(p->b_scales_stride & 3);
    const bool wide_out = aligned_to(p->out, 4) && !((p->n | p->out_stride | (contract ? p->out_matrix_stride : 0)) & 1);
    const ProductArgs a{p->a_scales_stride, p->b_scales_stride, p->b_scales_matrix_stride, p->out_stride, p->out_matrix_stride,
                        p->a_scales, p->b_scales, p->starts, p->status, (uint32_t)p->m, (uint32_t)p->n, (uint32_t)p->k, p->n_experts,
                        words_a, words_b, p->b_blocks, wide_out, tile_m};
    if (!encode_tiled()) return record_cuda_error(cudaErrorNotSupported);
    CUtensorMap am, bm;
    if (!operand_map(&am, p->a, p->k, p->m, 1, p->a_stride, 0, 64) ||
        !operand_map(&bm, p->b, p->k, p->n, rows ? p->n_experts : 1, p->b_stride, p->b_matrix_stride, 128))
        return record_cuda_error(cudaErrorInvalidValue);
    cudaError_t e = cudaSuccess;
    with_dtype(p->out_dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto mode_c) {
            constexpr int MODE = decltype(mode_c)::value;
            e = launch_product<MODE, DT>(a, am, bm, p->out, grid, dev, (cudaStream_t)stream);
        };
        if (rows) go(std::integral_constant<int, CIERA_PRODUCT_ROWS>());
        else if (contract) go(std::integral_constant<int, CIERA_PRODUCT_CONTRACT>());
        else go(std::integral_constant<int, CIERA_PRODUCT_DENSE>());
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
