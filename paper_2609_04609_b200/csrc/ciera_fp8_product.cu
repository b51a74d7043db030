// Products of e4m3 operands with a power of two for each block of 128 values of the contraction.
//
// out = sum over blocks b of 2^(sa + sb) * a_b * b_b^T.  The tensor cores take a power of two for each row and 32 values
// (kind::mxf8f6f4), so a block's scale is handed to them four times over and the sum over all blocks stays in tensor memory in
// fp32: no result passes through registers before the last block.
//
// One persistent block of threads per SM takes tiles of 128 rows x BN columns:
//   warp 0      copies tiles of a and b (128 values of the contraction) into a ring of stages by tensor maps
//   warp 1      copies a stage's scales into tensor memory and starts its four products
//   warps 2, 3  read the scale bytes, a stage each in turn, and lay them out as the tensor cores want them: row r's byte four
//               times over in word r / 32 of line r % 32
//   warps 4-7   read finished sums, round them and write them, 128 bytes of a row at a time through shared memory
// Two sums are in flight, so a tile's products run while the one before is written.  Tensor memory has 512 columns: with
// BN = 256 the two sums share 64 columns, which are the first that are read (the next tile's products wait for them alone),
// and 64 columns hold the scales, a slot for each stage.
#include <cuda.h>

#include <type_traits>

#include "ciera_numeric.cuh"
#include "ciera_tensor.cuh"

namespace ciera {

constexpr int kProductThreads = 256;
constexpr int kStages = 4;
constexpr uint32_t kTileM = 128;
constexpr uint32_t kMaxSegments = 1024;

struct ProductArgs {
    uint64_t a_scales_stride, b_scales_stride, b_scales_matrix_stride, out_stride, out_matrix_stride;
    const uint8_t* a_scales;
    const uint8_t* b_scales;
    const int32_t* starts;
    int32_t* status;
    uint32_t m, n, k, n_experts;
    int32_t a_words, b_words;  // scale bytes of rows may be read four at a time
    int32_t b_blocks;
    int32_t wide_out;  // rows of out start at multiples of 16 bytes
};

template <int BN>
struct alignas(1024) ProductSmem {
    uint8_t a[kStages][kTileM * 128];
    uint8_t b[kStages][BN * 128];
    uint4 a_scales[kStages][32];
    uint4 b_scales[kStages][BN / 128][32];
    uint4 out[4][32 * 8];  // 32 rows of 128 bytes of each writing warp
    uint64_t full[kStages], empty[kStages], sums_full[2], sums_free[2], done;
    uint32_t tmem;
    int abort;
    int32_t starts[kMaxSegments + 1];
};

// Where a sum and the scales of a stage are in tensor memory.
template <int BN>
__device__ __forceinline__ uint32_t sum_column(uint32_t which) { return which * (BN == 256 ? 192 : 128); }
template <int BN>
__device__ __forceinline__ uint32_t scales_column(uint32_t stage) { return (BN == 256 ? 448 : 256) + 16 * stage; }

// The tiles of a block of threads, in order, and the blocks of the contraction in each.
template <int MODE, int BN>
struct Walk {
    const ProductArgs& p;
    const int32_t* starts;
    uint32_t n_tiles, m_tiles, all, at;
    uint32_t e = 0, m0 = 0, n0 = 0, m1 = 0, kb0 = 0, kb1 = 0;

    __device__ Walk(const ProductArgs& p_, const int32_t* starts_) : p(p_), starts(starts_), at(blockIdx.x) {
        n_tiles = (p.n + BN - 1) / BN;
        m_tiles = MODE == CIERA_PRODUCT_ROWS ? (uint32_t)starts[p.n_experts] / kTileM : (p.m + kTileM - 1) / kTileM;
        all = m_tiles * n_tiles * (MODE == CIERA_PRODUCT_CONTRACT ? p.n_experts : 1u);
    }
    __device__ bool next() {  // false behind the last tile
        if (at >= all) return false;
        const uint32_t row = at / n_tiles;
        n0 = (at - row * n_tiles) * BN;
        if (MODE == CIERA_PRODUCT_CONTRACT) {
            e = row / m_tiles;
            m0 = (row - e * m_tiles) * kTileM;
            m1 = p.m;
            kb0 = (uint32_t)starts[e] / 128;
            kb1 = (uint32_t)starts[e + 1] / 128;
        } else {
            m0 = row * kTileM;
            m1 = p.m;
            if (MODE == CIERA_PRODUCT_ROWS)
                while ((uint32_t)starts[e + 1] <= m0) ++e;  // (tiles come in rising order)
            kb0 = 0;
            kb1 = (p.k + 127) / 128;
        }
        at += gridDim.x;
        return true;
    }
};

// 128 scale bytes of a block, four rows a lane: rows row0 + 4 * lane ...; rows from `rows` on count as 1
__device__ __forceinline__ uint32_t row_scales(const uint8_t* line, uint32_t row0, uint32_t rows, bool words, int lane) {
    const uint32_t r = row0 + 4 * lane;
    if (words && r + 3 < rows) return __ldg(reinterpret_cast<const uint32_t*>(line + r));
    uint32_t v = 0x7f7f7f7fu;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (r + i < rows) v = (v & ~(255u << (8 * i))) | (uint32_t)__ldg(line + r + i) << (8 * i);
    return v;
}
// ... as the tensor cores want them: line `lane` has rows lane, 32 + lane, 64 + lane, 96 + lane
__device__ __forceinline__ uint4 spread_scales(uint32_t four, int lane) {
    const uint32_t pick = 0x1111u * (lane & 3);
    uint4 v;
    v.x = __byte_perm(__shfl_sync(~0u, four, lane >> 2), 0, pick);
    v.y = __byte_perm(__shfl_sync(~0u, four, 8 + (lane >> 2)), 0, pick);
    v.z = __byte_perm(__shfl_sync(~0u, four, 16 + (lane >> 2)), 0, pick);
    v.w = __byte_perm(__shfl_sync(~0u, four, 24 + (lane >> 2)), 0, pick);
    return v;
}

// 32 columns of 16-byte units: `units` of them hold the sums of 64 (16-bit types) or 32 columns, rounded
template <int DT>
__device__ __forceinline__ uint4 pack_unit(const uint32_t* r) {
    if constexpr (DT == CIERA_FP32) {
        return make_uint4(r[0], r[1], r[2], r[3]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = __uint_as_float(r[2 * i]), hi = __uint_as_float(r[2 * i + 1]);
            if constexpr (DT == CIERA_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __half2 h = __floats2half2_rn(lo, hi);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Writes 128 bytes of each of the warp's 32 rows: `unit(u)` gives the lane's row's unit u.  `stage`: 4 KB of the warp's own.
template <int DT, class F>
__device__ __forceinline__ void write_rows(F&& unit, uint4* stage, value_t<DT>* out, uint64_t stride, uint32_t rows_left, uint32_t col,
                                           uint32_t n, bool wide, int lane) {
    constexpr uint32_t V = 16 / sizeof(value_t<DT>);
    __syncwarp();
#pragma unroll
    for (int u = 0; u < 8; ++u) stage[lane * 8 + (u ^ (lane & 7))] = unit(u);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = 4 * i + (lane >> 3), u = lane & 7, c = col + u * V;
        if (r >= rows_left || c >= n) continue;
        const uint4 v = stage[r * 8 + (u ^ (r & 7))];
        value_t<DT>* to = out + r * stride + c;
        if (wide && c + V <= n) {
            *reinterpret_cast<uint4*>(to) = v;
        } else {
            const Pack<value_t<DT>, (int)V> w = *reinterpret_cast<const Pack<value_t<DT>, (int)V>*>(&v);
#pragma unroll
            for (uint32_t q = 0; q < V; ++q)
                if (c + q < n) to[q] = w.v[q];
        }
    }
}

template <int MODE, int DT, int BN>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const ProductArgs p, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                   value_t<DT>* __restrict__ out) {
    extern __shared__ uint8_t product_smem[];
    ProductSmem<BN>& sm = *reinterpret_cast<ProductSmem<BN>*>(product_smem + (-smem_u32(product_smem) & 1023u));
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 2);  // the copies' thread and the scales' warp
            mbar_init(&sm.empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.sums_full[i], 1);
            mbar_init(&sm.sums_free[i], 4);
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
    tensor_fence_after();
    const uint32_t tmem = sm.tmem;
    if (bad) {
        if (p.status && threadIdx.x == 0) atomicCAS(p.status, 0, (int32_t)CIERA_ERR_CORRUPT);
        if (warp == 1) tmem_free(tmem, 512);
        return;
    }
    Walk<MODE, BN> w(p, sm.starts);
    volatile int* abort = &sm.abort;
    uint32_t it = 0;  // blocks of the contraction so far

    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            while (ok && w.next()) {
                for (uint32_t kb = w.kb0; kb < w.kb1; ++kb, ++it) {
                    const uint32_t s = it % kStages;
                    if (!mbar_wait(&sm.empty[s], ((it / kStages) & 1) ^ 1, abort, p.status)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(&sm.full[s], kTileM * 128 + BN * 128);
                    map_load2(sm.a[s], &a_map, (int32_t)(kb * 128), (int32_t)w.m0, &sm.full[s]);
                    map_load3(sm.b[s], &b_map, (int32_t)(kb * 128), (int32_t)w.n0, MODE == CIERA_PRODUCT_ROWS ? (int32_t)w.e : 0, &sm.full[s]);
                }
            }
            // given up: the copies in flight end before the block does
            if (!ok)
                for (uint32_t i = it < kStages ? 0 : it - kStages; i < it; ++i) {
                    int none = 0;
                    mbar_wait(&sm.full[i % kStages], (i / kStages) & 1, &none, p.status, 1024);
                }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t instruction = mx_instruction(kTileM, BN);
            uint32_t tile = 0;
            bool ok = true;
            while (ok && w.next()) {
                if (w.kb0 == w.kb1) continue;
                // BN = 128: the sum before the last one has been read.  BN = 256: the columns shared with the last one have.
                if (BN == 256 ? tile >= 1 : tile >= 2) {
                    const uint32_t of = tile - (BN == 256 ? 1 : 2);
                    if (!mbar_wait(&sm.sums_free[of & 1], (of >> 1) & 1, abort, p.status)) break;
                    tensor_fence_after();
                }
                const uint32_t d = tmem + sum_column<BN>(tile & 1);
                for (uint32_t kb = w.kb0; kb < w.kb1; ++kb, ++it) {
                    const uint32_t s = it % kStages;
                    if (!mbar_wait(&sm.full[s], (it / kStages) & 1, abort, p.status)) {
                        ok = false;
                        break;
                    }
                    tensor_fence_after();
                    const uint32_t sc = tmem + scales_column<BN>(s);
                    tmem_copy_scales(sc, scales_descriptor(sm.a_scales[s]));
#pragma unroll
                    for (int h = 0; h < BN / 128; ++h) tmem_copy_scales(sc + 8 + 4 * h, scales_descriptor(sm.b_scales[s][h]));
                    const uint64_t da = operand_descriptor(sm.a[s]), db = operand_descriptor(sm.b[s]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) tensor_mma_mx(d, da + 2 * j, db + 2 * j, instruction, sc, sc + 8, kb > w.kb0 || j > 0);
                    tensor_commit(&sm.empty[s]);
                }
                if (ok) tensor_commit(&sm.sums_full[tile & 1]);
                ++tile;
            }
            // nothing of this thread's is in flight when the tensor memory is given back
            tensor_commit(&sm.done);
            int none = 0;
            mbar_wait(&sm.done, 0, &none, p.status);
        }
        __syncwarp();
    } else if (warp < 4) {
        // this warp's blocks are every other one; the bytes of the next are fetched before it waits for room for the last
        uint32_t kb = 0;
        bool more = true, some = false;
        auto advance = [&](uint32_t by) {
            while (by) {
                if (some && kb + 1 < w.kb1) {
                    ++kb, --by;
                    continue;
                }
                do {
                    if (!w.next()) {
                        more = false;
                        return;
                    }
                } while (w.kb0 == w.kb1);
                some = true;
                kb = w.kb0;
                --by;
            }
        };
        uint32_t va, vb[BN / 128];
        auto fetch = [&]() {
            va = row_scales(p.a_scales + kb * p.a_scales_stride, w.m0, w.m1, p.a_words, lane);
#pragma unroll
            for (int h = 0; h < BN / 128; ++h) {
                const uint32_t n0 = w.n0 + 128 * h;
                if (p.b_blocks)
                    vb[h] = n0 < p.n ? __ldg(p.b_scales + (MODE == CIERA_PRODUCT_ROWS ? w.e : 0) * p.b_scales_matrix_stride +
                                             (uint64_t)(n0 / 128) * p.b_scales_stride + kb) * 0x01010101u
                                     : 0x7f7f7f7fu;
                else
                    vb[h] = row_scales(p.b_scales + kb * p.b_scales_stride, n0, p.n, p.b_words, lane);
            }
        };
        it = warp - 2;
        advance(1 + it);
        if (more) fetch();
        while (more) {
            const uint32_t s = it % kStages, turn = it / kStages;
            const uint4 sa = spread_scales(va, lane);
            uint4 sb[BN / 128];
#pragma unroll
            for (int h = 0; h < BN / 128; ++h) sb[h] = p.b_blocks ? make_uint4(vb[h], vb[h], vb[h], vb[h]) : spread_scales(vb[h], lane);
            it += 2;
            advance(2);
            if (more) fetch();
            if (!mbar_wait(&sm.empty[s], (turn & 1) ^ 1, abort, p.status)) break;
            sm.a_scales[s][lane] = sa;
#pragma unroll
            for (int h = 0; h < BN / 128; ++h) sm.b_scales[s][h][lane] = sb[h];
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.full[s]);
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3;
        uint4* stage = sm.out[quarter];
        uint32_t tile = 0;
        while (w.next()) {
            const uint32_t m = w.m0 + quarter * 32;
            const uint32_t rows_left = m < w.m1 ? w.m1 - m : 0;
            value_t<DT>* o = out + (MODE == CIERA_PRODUCT_CONTRACT ? w.e * p.out_matrix_stride : 0) + m * p.out_stride;
            if (w.kb0 == w.kb1) {  // nothing to add up
                for (uint32_t c = 0; c < BN; c += 128 / sizeof(value_t<DT>))
                    write_rows<DT>([&](int) { return make_uint4(0, 0, 0, 0); }, stage, o, p.out_stride, rows_left, w.n0 + c, p.n, p.wide_out, lane);
                continue;
            }
            const uint32_t which = tile & 1;
            if (!mbar_wait(&sm.sums_full[which], (tile >> 1) & 1, abort, p.status, kMaxBarrierPolls + (w.kb1 - w.kb0))) break;
            __syncwarp();
            tensor_fence_after();
            const uint32_t from = tmem + ((uint32_t)quarter << 21) + sum_column<BN>(which);
            constexpr int kParts = BN / 64;
            for (int i = 0; i < kParts; ++i) {
                // the columns shared with the other sum first
                const uint32_t c = BN == 256 && which == 0 ? ((i + 3) & 3) * 64 : i * 64;
                uint32_t r[2][32];
                tmem_load32(from + c, r[0]);
                tmem_load32(from + c + 32, r[1]);
                tmem_wait_load();
                if (BN == 256 ? i == 0 : i == kParts - 1) {
                    tensor_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.sums_free[which]);
                }
                if constexpr (DT == CIERA_FP32) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        write_rows<DT>([&](int u) { return pack_unit<DT>(r[h] + 4 * u); }, stage, o, p.out_stride, rows_left,
                                       w.n0 + c + 32 * h, p.n, p.wide_out, lane);
                } else {
                    write_rows<DT>([&](int u) { return pack_unit<DT>(r[u >> 2] + 8 * (u & 3)); }, stage, o, p.out_stride, rows_left,
                                   w.n0 + c, p.n, p.wide_out, lane);
                }
            }
            ++tile;
        }
        __syncwarp();
    }
    tensor_fence_before();
    __syncthreads();
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
    return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, matrices ? 3 : 2, const_cast<void*>(p), dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_count(int* n) {
    static std::atomic<int> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (dev < 64 && (*n = known[dev].load(std::memory_order_relaxed)) > 0) return CIERA_OK;
    e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (dev < 64) known[dev].store(*n, std::memory_order_relaxed);
    return CIERA_OK;
}

template <int MODE, int DT, int BN>
static cudaError_t launch_product(const ProductArgs& a, const CUtensorMap& am, const CUtensorMap& bm, void* out, uint32_t grid, cudaStream_t s) {
    constexpr size_t smem = sizeof(ProductSmem<BN>) + 1024;  // (the ring starts at a multiple of 1024)
    auto kernel = product_kernel<MODE, DT, BN>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_after(kernel, dim3(grid), kProductThreads, smem, s, a, am, bm, (value_t<DT>*)out);
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
    int sms = 0;
    const int rc = sm_count(&sms);
    if (rc) return rc;
    // tiles of 256 columns read a third less than two of 128; narrower ones where the wide ones would leave SMs without work
    const uint64_t mt = (p->m + kTileM - 1) / kTileM, groups = contract ? p->n_experts : 1;
    const uint64_t wide = mt * ((p->n + 255) / 256) * groups, narrow = mt * nb * groups;
    const bool bn256 = wide >= (uint64_t)sms;
    if (narrow > 0xffffffffull - 65536) return CIERA_ERR_UNSUPPORTED;
    const uint64_t tiles = bn256 ? wide : narrow;
    const uint32_t grid = (uint32_t)(tiles < (uint64_t)sms ? tiles : sms);
    const uint64_t v = dtype_bytes(p->out_dtype);
    const bool words_a = aligned_to(p->a_scales, 4) && !(p->a_scales_stride & 3), words_b = aligned_to(p->b_scales, 4) && !(p->b_scales_stride & 3);
    const bool wide_out = aligned_to(p->out, 16) && !(p->out_stride * v & 15) && (!contract || !(p->out_matrix_stride * v & 15));
    const ProductArgs a{p->a_scales_stride, p->b_scales_stride, p->b_scales_matrix_stride, p->out_stride, p->out_matrix_stride,
                        p->a_scales, p->b_scales, p->starts, p->status, (uint32_t)p->m, (uint32_t)p->n, (uint32_t)p->k, p->n_experts,
                        words_a, words_b, p->b_blocks, wide_out};
    if (!encode_tiled()) return record_cuda_error(cudaErrorNotSupported);
    CUtensorMap am, bm;
    if (!operand_map(&am, p->a, p->k, p->m, 0, p->a_stride, 0, kTileM) ||
        !operand_map(&bm, p->b, p->k, p->n, rows ? p->n_experts : 1, p->b_stride, p->b_matrix_stride, bn256 ? 256 : 128))
        return record_cuda_error(cudaErrorInvalidValue);
    cudaError_t e = cudaSuccess;
    with_dtype(p->out_dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto mode_c) {
            constexpr int MODE = decltype(mode_c)::value;
            e = bn256 ? launch_product<MODE, DT, 256>(a, am, bm, p->out, grid, (cudaStream_t)stream)
                      : launch_product<MODE, DT, 128>(a, am, bm, p->out, grid, (cudaStream_t)stream);
        };
        if (rows) go(std::integral_constant<int, CIERA_PRODUCT_ROWS>());
        else if (contract) go(std::integral_constant<int, CIERA_PRODUCT_CONTRACT>());
        else go(std::integral_constant<int, CIERA_PRODUCT_DENSE>());
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
