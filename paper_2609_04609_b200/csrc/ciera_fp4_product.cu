// Products of e2m1 operands with a power of two for each row and 32 values of the contraction.
//
// out = sum over groups of 2^(sa + sb) * a_g * b_g^T.  The tensor cores take such operands as they are (kind::mxf4, 64 values of
// the contraction an instruction, at twice the rate of 8 bits) and apply the scales themselves; the sum over the whole contraction
// stays in tensor memory in fp32.
//
// Persistent pairs of blocks of threads (a cluster on two SMs) take tiles of 256 columns x 256 (or 128) rows of out, as the 8-bit
// products do and for the same reason: b's rows are the first operand, 128 to a block, a's rows the second, half of them to a
// block, and segments of a's end at any multiple of 128.  A stage is 128 bytes of every row, 256 values of the contraction, and the
// two atoms of scales of each 128 rows that go with them: an atom is laid out as tensor memory wants it (row r's four bytes in
// word r / 32 of line r % 32), so it is copied there from where the tensor map has put it, and no thread touches a scale.
//   warp 0      copies tiles and scales into a ring of stages by tensor maps
//   warp 1      of the first block: copies a stage's scales into tensor memory and starts its four products
//   warps 2-5   read finished sums (a lane is a column of out) and write them
// Two sums are in flight.  Tensor memory has 512 columns: the two sums share 128, and the last 128 hold the scales of five stages.
//
// Measured: 8192^3 174 to 177 us, 6.3 PFLOP/s, in a short run (208 us back to back, where the clock falls with the power); 32768 rows of
// 64 experts, 2048 x 2048, 79 us, 64 without writing the results (97 back to back); one token on 8 experts 9.6 us, of which DRAM needs 3.
#include <type_traits>

#include "ciera_product.cuh"

namespace ciera {

constexpr int kProduct4Threads = 192;
constexpr int kStages4 = 6;
constexpr uint32_t kTile4N = 256;  // columns of a pair's tile
constexpr uint32_t kStageK = 256;  // values of the contraction in a stage
constexpr uint32_t kMaxSegments4 = 1024;
constexpr uint32_t kShared4 = 128, kSecondSum4 = 256 - kShared4, kScalesAt4 = kSecondSum4 + 256;  // columns of tensor memory
constexpr uint32_t kScaleColumns = 24;  // of a stage: two atoms of b's rows, two of each 128 of a's
constexpr uint32_t kScaleStages = 5;    // that tensor memory holds the scales of
static_assert(kScalesAt4 + kScaleStages * kScaleColumns <= 512 && kScaleStages < kStages4, "not in tensor memory");

struct Product4Args {
    uint64_t out_stride;
    const int32_t* starts;
    int32_t* status;
    uint32_t m, n, k, n_experts;
    int32_t wide_out;  // 16-bit columns of out may be written two at a time
    uint32_t tile_m;   // rows of a tile: 256 or 128
};

struct alignas(1024) Product4Smem {
    uint8_t b[kStages4][128 * 128];
    uint8_t a[kStages4][128 * 128];
    uint8_t b_scales[kStages4][2][512];     // [atom of the contraction]
    uint8_t a_scales[kStages4][2][2][512];  // [128 rows][atom of the contraction]
    uint64_t full[kStages4], empty[kStages4], sums_full[2], sums_free[2], done;
    uint32_t tmem;
    int abort;
    int32_t starts[kMaxSegments4 + 1];
    uint32_t first_tile[kMaxSegments4 + 1];  // rows' tiles before each segment
};
constexpr uint32_t kScaleBytes4 = 6 * 512;  // of a stage, in each block
static_assert(sizeof(Product4Smem) + 1024 <= 227 * 1024, "more than a block may have");

// The tiles of a pair, in order.
template <bool ROWS>
struct Walk4 {
    const Product4Args& p;
    const Product4Smem& sm;
    uint32_t n_tiles, all, at;
    uint32_t e = 0, m0 = 0, n0 = 0, m1 = 0;

    __device__ Walk4(const Product4Args& p_, const Product4Smem& sm_) : p(p_), sm(sm_), at(blockIdx.x >> 1) {
        n_tiles = (p.n + kTile4N - 1) / kTile4N;
        all = (ROWS ? sm.first_tile[p.n_experts] : (p.m + p.tile_m - 1) / p.tile_m) * n_tiles;
    }
    __device__ bool next() {  // false behind the last tile
        if (at >= all) return false;
        const uint32_t row = at / n_tiles;
        n0 = (at - row * n_tiles) * kTile4N;
        if (ROWS) {
            while (sm.first_tile[e + 1] <= row) ++e;  // (tiles come in rising order)
            m0 = (uint32_t)sm.starts[e] + (row - sm.first_tile[e]) * p.tile_m;
            m1 = (uint32_t)sm.starts[e + 1];
        } else {
            m0 = row * p.tile_m;
            m1 = p.m;
        }
        at += gridDim.x >> 1;
        return true;
    }
    // rows of the tile that the products are made for
    __device__ uint32_t height() const { return m1 - m0 > 128 && p.tile_m == 256 ? 256u : 128u; }
};

template <bool ROWS, int DT>
__global__ void __launch_bounds__(kProduct4Threads, 1)
    product4_kernel(const Product4Args p, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                    const __grid_constant__ CUtensorMap as_map, const __grid_constant__ CUtensorMap bs_map, value_t<DT>* __restrict__ out) {
    extern __shared__ uint8_t product_smem[];
    Product4Smem& sm = *reinterpret_cast<Product4Smem*>(product_smem + (-smem_u32(product_smem) & 1023u));
    const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, (int)(threadIdx.x >> 5), 0);
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        prefetch_map(&as_map);
        prefetch_map(&bs_map);
        for (int s = 0; s < kStages4; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.empty[s], 1);
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
    if (ROWS) {
        for (uint32_t i = threadIdx.x; i <= p.n_experts; i += kProduct4Threads) {
            const int32_t v = p.starts[i], before = i ? p.starts[i - 1] : 0;
            sm.starts[i] = v;
            bad |= v < before || (v & 127) || (uint32_t)v > p.m || (i == 0 && v != 0);
        }
    }
    bad = __syncthreads_or(bad);
    if (ROWS && !bad && warp == 0) {
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
    tensor_fence_before();
    cluster_sync();  // barriers, tables and tensor memory of both blocks are there
    tensor_fence_after();
    const uint32_t tmem = sm.tmem;
    if (bad) {  // (in both blocks: they read the same table)
        if (p.status && threadIdx.x == 0 && rank == 0) atomicCAS(p.status, 0, (int32_t)CIERA_ERR_CORRUPT);
        if (warp == 1) tmem_free(tmem, 512);
        return;
    }
    Walk4<ROWS> w(p, sm);
    volatile int* abort = &sm.abort;
    const uint32_t stages = (p.k + kStageK - 1) / kStageK;  // of a tile

    if (warp == 0) {
        bool ok = true;
        uint32_t it = 0, s = 0, odd = 1;  // stages so far, the next one, and the parity of its last phase
        while (ok && w.next()) {
            const uint32_t half = w.height() / 2;
            const int32_t m0 = (int32_t)(w.m0 + rank * half), n0 = (int32_t)(w.n0 + rank * 128);
            for (uint32_t kb = 0; kb < stages; ++kb, ++it) {
                if (!mbar_wait_soon(&sm.empty[s], odd, abort, p.status)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx(&sm.full[s], 2 * (128 * 128 + half * 128 + kScaleBytes4));
                    const uint32_t full = in_first_block(&sm.full[s]);
                    const int32_t k0 = (int32_t)(kb * 128), atom = (int32_t)(kb * 2);
                    map_load3(sm.b[s], &b_map, k0, n0, ROWS ? (int32_t)w.e : 0, full);
                    map_load3(sm.a[s], &a_map, k0, m0, 0, full);
                    if (half == 128) map_load3(sm.a[s] + 64 * 128, &a_map, k0, m0 + 64, 0, full);
                    map_load4(sm.b_scales[s], &bs_map, 0, atom, n0 / 128, ROWS ? (int32_t)w.e : 0, full);
                    map_load4(sm.a_scales[s], &as_map, 0, atom, (int32_t)(w.m0 / 128), 0, full);
                }
                __syncwarp();
                if (++s == kStages4) s = 0, odd ^= 1;
            }
        }
        // No block leaves while an arrival is on its way to one of its barriers: those that nobody else waits for are waited for
        // here, and with them all products that read the stages.
        const uint32_t since = it < kStages4 ? 0 : it - kStages4;
        if (ok) {
            for (uint32_t i = since; i < it; ++i) mbar_wait_soon(&sm.empty[i % kStages4], (i / kStages4) & 1, abort, p.status);
        } else if (rank == 0 && lane == 0) {  // given up: the copies in flight (they report to the first block) end before the cluster does
            for (uint32_t i = since; i < it; ++i) {
                int none = 0;
                mbar_wait(&sm.full[i % kStages4], (i / kStages4) & 1, &none, p.status, 1024);
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
            uint32_t tile = 0, it = 0, s = 0, odd = 0;
            bool ok = true;
            const uint64_t db0 = operand_descriptor(sm.b[0]), da0 = operand_descriptor(sm.a[0]);
            while (ok && w.next()) {
                if (tile) {  // the columns shared with the sum before have been read
                    if (!mbar_wait_cluster(&sm.sums_free[(tile - 1) & 1], ((tile - 1) >> 1) & 1, abort, p.status)) break;
                    tensor_fence_after();
                }
                const uint32_t instruction = mx4_instruction(256, w.height()), d = tmem + (tile & 1) * kSecondSum4;
                for (uint32_t kb = 0; kb < stages; ++kb) {
                    // (the products whose scales these replace have ended: those of two stages ago, with room for two, held up the rest:
                    // 8192^3 176 us in a short run, 172 so; no difference back to back)
                    if (!mbar_wait_soon(&sm.full[s], odd, abort, p.status) ||
                        (it >= kScaleStages && !mbar_wait_soon(&sm.empty[(it - kScaleStages) % kStages4], ((it - kScaleStages) / kStages4) & 1, abort, p.status))) {
                        ok = false;
                        break;
                    }
                    tensor_fence_after();
                    const bool last = kb + 1 == stages;
                    const uint32_t left = min(p.k - kb * kStageK, kStageK);
                    // b's scales, then a's: both halves of a's rows of an atom side by side
                    const uint32_t sc = tmem + kScalesAt4 + it % kScaleStages * kScaleColumns;
                    if (elect_one()) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            tmem_copy_scales(sc + 12 * i, scales_descriptor(sm.b_scales[s][i]));
                            tmem_copy_scales(sc + 12 * i + 4, scales_descriptor(sm.a_scales[s][0][i]));
                            tmem_copy_scales(sc + 12 * i + 8, scales_descriptor(sm.a_scales[s][1][i]));
                        }
                        const uint64_t db = db0 + s * (128 * 128 / 16), da = da0 + s * (128 * 128 / 16);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (i * 64 < left)
                                tensor_mma_mx4(d, db + 2 * i, da + 2 * i, instruction + (i & 1) * mx_byte(2), sc + 12 * (i >> 1), sc + 12 * (i >> 1) + 4,
                                               kb > 0 || i > 0);
                        tensor_commit(&sm.empty[s]);
                        if (last) tensor_commit(&sm.sums_full[tile & 1]);
                    }
                    __syncwarp();
                    ++it;
                    if (++s == kStages4) s = 0, odd ^= 1;
                }
                ++tile;
            }
            // nothing that this warp started is in flight when the tensor memory is given back
            if (elect_one()) tensor_commit(&sm.done);
            int none = 0;
            mbar_wait_soon(&sm.done, 0, &none, p.status);
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3;
        uint32_t tile = 0;
        while (w.next()) {
            const uint32_t n = w.n0 + rank * 128 + quarter * 32;
            auto write = [&](const uint32_t(&r)[32], uint32_t part) {
                write_part<DT>(r, out, p.out_stride, w.m0 + 32 * part, w.m1, n + lane, p.n, p.wide_out, lane);
            };
            const uint32_t parts = w.height() / 32, which = tile & 1;
            if (!mbar_wait_soon(&sm.sums_full[which], (tile >> 1) & 1, abort, p.status, kMaxBarrierPolls + stages)) break;
            __syncwarp();
            tensor_fence_after();
            const uint32_t from = tmem + ((uint32_t)quarter << 21) + which * kSecondSum4;
            // the columns shared with the other sum first: the second's first four parts, the first's last four of eight
            const uint32_t first = which == 0 && parts == 8 ? 4 : 0;
            uint32_t r[4][32];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_load32(from + 32 * (first + i), r[i]);
            tmem_wait_load();
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_read(in_first_block(&sm.sums_free[which]));
#pragma unroll
            for (int i = 0; i < 4; ++i) write(r[i], first + i);
            for (uint32_t i = 4; i < parts; ++i) {
                const uint32_t part = first ? i - 4 : i;
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

// `lines` lines of atoms for each of `matrices` matrices; boxes of two atoms of `box` lines
static bool scales_map(CUtensorMap* map, const void* p, uint64_t atoms, uint64_t lines, uint64_t matrices, uint64_t stride,
                       uint64_t matrix_stride, uint32_t box) {
    if (lines <= 1) stride = atoms * 512;  // (never stepped by)
    if (matrices <= 1) matrix_stride = lines * stride;
    const cuuint64_t dims[4] = {128, atoms, lines, matrices}, strides[3] = {512, stride, matrix_stride};
    const cuuint32_t boxes[4] = {128, 2, box, 1}, steps[4] = {1, 1, 1, 1};
    return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, const_cast<void*>(p), dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Product4Maps {
    CUtensorMap a, b, a_scales, b_scales;
};

template <bool ROWS, int DT>
static cudaError_t launch_product4(const Product4Args& a, const Product4Maps& maps, void* out, uint32_t pairs, int dev, cudaStream_t s) {
    static std::atomic<uint64_t> allowed{0};  // devices on which this instance may have its shared memory
    constexpr size_t smem = sizeof(Product4Smem) + 1024;  // (the ring starts at a multiple of 1024)
    auto kernel = product4_kernel<ROWS, DT>;
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
    cfg.blockDim = dim3(kProduct4Threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, maps.a, maps.b, maps.a_scales, maps.b_scales, (value_t<DT>*)out);
}

}  // namespace ciera

using namespace ciera;

extern "C" int ciera_fp4_matmul(const ciera_fp4_product* p, void* stream) {
    if (!p || (p->mode != CIERA_PRODUCT_DENSE && p->mode != CIERA_PRODUCT_ROWS)) return CIERA_ERR_INVALID_ARG;
    if (p->out_dtype != CIERA_BF16 && p->out_dtype != CIERA_FP32 && p->out_dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    const bool rows = p->mode == CIERA_PRODUCT_ROWS;
    if (p->m < 1 || p->n < 1 || p->k < 1 || p->m > kMaxExtent || p->n > kMaxExtent || p->k > kMaxExtent) return CIERA_ERR_INVALID_ARG;
    const uint64_t line = (p->k + 1) / 2, atoms = (p->k + 127) / 128;
    if (!p->a || !p->a_scales || !p->b || !p->b_scales || !p->out || rows != (p->starts != nullptr) ||
        (rows && (p->n_experts < 1 || p->n_experts > kMaxSegments4)) || (p->m > 1 && p->a_stride < line) || (p->n > 1 && p->b_stride < line) ||
        (p->m > 128 && p->a_scales_stride < atoms * 512) || (p->n > 128 && p->b_scales_stride < atoms * 512) || (p->m > 1 && p->out_stride < p->n))
        return CIERA_ERR_INVALID_ARG;
    // (strides of single rows and matrices count for nothing)
    const bool several = rows && p->n_experts > 1;
    if (!aligned_to(p->a, 16) || !aligned_to(p->b, 16) || !aligned_to(p->a_scales, 16) || !aligned_to(p->b_scales, 16) ||
        (p->m > 1 && (p->a_stride & 15)) || (p->n > 1 && (p->b_stride & 15)) || (several && ((p->b_matrix_stride | p->b_scales_matrix_stride) & 15)) ||
        (p->m > 128 && (p->a_scales_stride & 511)) || (p->n > 128 && (p->b_scales_stride & 511)) || !aligned_to(p->out, dtype_bytes(p->out_dtype)) ||
        !aligned_to(p->starts, 4) || !aligned_to(p->status, 4))
        return CIERA_ERR_MISALIGNED;
    const uint64_t most = 1ull << 40;
    if ((p->m > 1 && p->a_stride >= most) || (p->n > 1 && p->b_stride >= most) || (several && (p->b_matrix_stride >= most || p->b_scales_matrix_stride >= most)) ||
        (p->m > 128 && p->a_scales_stride >= most) || (p->n > 128 && p->b_scales_stride >= most))
        return CIERA_ERR_UNSUPPORTED;
    int dev = 0, sms = 0;
    const int rc = device_and_sms(&dev, &sms);
    if (rc) return rc;
    // tiles of 128 rows where those of 256 would leave SMs without work (every segment has at most one more than its rows fill)
    const uint64_t n_tiles = (p->n + kTile4N - 1) / kTile4N, pairs = sms / 2;
    const auto tiles_of = [&](uint64_t h) { return ((p->m + h - 1) / h) * n_tiles; };
    const uint32_t tile_m = tiles_of(256) >= pairs ? 256 : 128;
    const uint64_t tiles = tiles_of(tile_m) + (rows && tile_m == 256 ? p->n_experts * n_tiles : 0);
    if (tiles > 0xffffffffull - 65536) return CIERA_ERR_UNSUPPORTED;
    const uint32_t grid = (uint32_t)(tiles < pairs ? tiles : pairs);
    const bool wide_out = aligned_to(p->out, 4) && !((p->n | p->out_stride) & 1);
    const Product4Args a{p->out_stride, p->starts, p->status, (uint32_t)p->m, (uint32_t)p->n, (uint32_t)p->k, p->n_experts, wide_out, tile_m};
    if (!encode_tiled()) return record_cuda_error(cudaErrorNotSupported);
    const uint64_t matrices = rows ? p->n_experts : 1;
    Product4Maps maps;
    if (!operand_map(&maps.a, p->a, line, p->m, 1, p->a_stride, 0, 64) ||
        !operand_map(&maps.b, p->b, line, p->n, matrices, p->b_stride, p->b_matrix_stride, 128) ||
        !scales_map(&maps.a_scales, p->a_scales, atoms, (p->m + 127) / 128, 1, p->a_scales_stride, 0, 2) ||
        !scales_map(&maps.b_scales, p->b_scales, atoms, (p->n + 127) / 128, matrices, p->b_scales_stride, p->b_scales_matrix_stride, 1))
        return record_cuda_error(cudaErrorInvalidValue);
    cudaError_t e = cudaSuccess;
    with_dtype(p->out_dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        e = rows ? launch_product4<true, DT>(a, maps, p->out, grid, dev, (cudaStream_t)stream)
                 : launch_product4<false, DT>(a, maps, p->out, grid, dev, (cudaStream_t)stream);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
