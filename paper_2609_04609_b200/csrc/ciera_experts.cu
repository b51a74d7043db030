// Slots in the order of the experts, and the weighted sum of a token's rows with its gradients.
#include <type_traits>

#include "ciera_numeric.cuh"

namespace ciera {

// ------------------------------------------------------------------------------------------ layout
// A stable counting sort.  The slots are cut into chunks of kLayoutChunk; a chunk's block counts its experts (layout_count),
// then every block adds up the chunks before its own and places its slots (layout_place); one chunk is placed at once.  Within a
// block each warp owns a stretch of neighbouring slots and a row of counters, so ranks come out in slot order whatever the
// order in which the counters are added to.  What a block waits for is the table of counts, so chunks are large: 262168 slots
// over 256 experts in chunks of 2048 took 27 us.
// That every block reads the counts of all chunks grows with the square of the slots, so from kLayoutScanFrom chunks on a launch
// in between (layout_scan) adds them up once: 1.2 million slots of 64 experts 19 us with it and 22 without, of 8 experts 20 and 16;
// 16 million of 256 experts 179 us and 1802.

constexpr int kLayoutWarps = 16;
constexpr int kLayoutRounds = 8;  // slots per lane
constexpr int kLayoutChunk = kLayoutWarps * kLayoutRounds * 32;
constexpr uint32_t kMaxExperts = 1024;
constexpr uint64_t kLayoutScanFrom = 256;
constexpr int kScanStretches = 32;

__device__ __forceinline__ void load_ids(const int32_t* __restrict__ experts, uint64_t n_slots, uint64_t base, int lane,
                                         uint32_t n_experts, uint32_t (&ids)[kLayoutRounds]) {
#pragma unroll
    for (int r = 0; r < kLayoutRounds; ++r) {
        const uint64_t i = base + r * 32 + lane;
        ids[r] = i < n_slots ? min((uint32_t)experts[i], n_experts) : n_experts;
    }
}

__global__ void __launch_bounds__(kLayoutWarps * 32) layout_count(const int32_t* __restrict__ experts, uint64_t n_slots,
                                                                  uint32_t n_experts, uint32_t* __restrict__ hist) {
    extern __shared__ uint32_t layout_smem[];
    for (uint32_t i = threadIdx.x; i < n_experts; i += blockDim.x) layout_smem[i] = 0;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t ids[kLayoutRounds];
    load_ids(experts, n_slots, (uint64_t)blockIdx.x * kLayoutChunk + warp * (kLayoutRounds * 32), lane, n_experts, ids);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kLayoutRounds; ++r)
        if (ids[r] < n_experts) atomicAdd(&layout_smem[ids[r]], 1u);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < n_experts; e += blockDim.x) hist[(uint64_t)blockIdx.x * n_experts + e] = layout_smem[e];
}

// In place of every chunk's counts those of the chunks before it, and behind the last chunk those of all.  A block has 32 experts, a
// warp a stretch of the chunks.
__global__ void __launch_bounds__(kScanStretches * 32) layout_scan(uint32_t* __restrict__ hist, uint32_t chunks, uint32_t n_experts) {
    __shared__ uint32_t sums[kScanStretches][32];
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    const uint32_t each = (chunks + kScanStretches - 1) / kScanStretches, begin = min(chunks, warp * each), end = min(chunks, begin + each);
    uint32_t sum = 0;
    if (e < n_experts) {
#pragma unroll 8
        for (uint32_t c = begin; c < end; ++c) sum += hist[(uint64_t)c * n_experts + e];
    }
    sums[warp][lane] = sum;
    __syncthreads();
    uint32_t run = 0;
    for (uint32_t w = 0; w < warp; ++w) run += sums[w][lane];
    if (e >= n_experts) return;
    for (uint32_t c = begin; c < end;) {
        uint32_t v[8];
        const uint32_t n = min(8u, end - c);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i] = i < n ? hist[(uint64_t)(c + i) * n_experts + e] : 0u;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            if (i < n) hist[(uint64_t)(c + i) * n_experts + e] = run;
            run += v[i];
        }
        c += n;
    }
    if (warp == kScanStretches - 1) hist[(uint64_t)chunks * n_experts + e] = run;
}

// hist: counts of every chunk, or NULL for a single chunk; SCANNED: as layout_scan leaves them
template <bool SCANNED>
__global__ void __launch_bounds__(kLayoutWarps * 32)
    layout_place(const int32_t* __restrict__ experts, uint64_t n_slots, uint32_t n_experts, const uint32_t* __restrict__ hist,
                 int32_t* __restrict__ starts, int32_t* __restrict__ counts, int32_t* __restrict__ row_of_slot,
                 int32_t* __restrict__ slot_of_row) {
    extern __shared__ uint32_t layout_smem[];
    uint32_t* before = layout_smem + kLayoutWarps * n_experts;  // slots of the chunks before this one
    uint32_t* total = before + n_experts;                       // of all chunks
    uint32_t* first = total + n_experts;                        // first row of the expert's segment (n_experts + 1)
    for (uint32_t i = threadIdx.x; i < (kLayoutWarps + 2) * n_experts; i += blockDim.x) layout_smem[i] = 0;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t base = (uint64_t)blockIdx.x * kLayoutChunk + warp * (kLayoutRounds * 32);
    uint32_t ids[kLayoutRounds];
    load_ids(experts, n_slots, base, lane, n_experts, ids);
    __syncthreads();
    uint32_t* next = layout_smem + warp * n_experts;
#pragma unroll
    for (int r = 0; r < kLayoutRounds; ++r)
        if (ids[r] < n_experts) atomicAdd(&next[ids[r]], 1u);
    if constexpr (SCANNED) {
        for (uint32_t e = threadIdx.x; e < n_experts; e += blockDim.x) {
            before[e] = hist[(uint64_t)blockIdx.x * n_experts + e];
            total[e] = hist[(uint64_t)gridDim.x * n_experts + e];
        }
    } else if (hist) {  // a thread for an expert and every so many chunks
        const uint32_t side = blockDim.x / n_experts > 1 ? blockDim.x / n_experts : 1;
        for (uint32_t i = threadIdx.x; i < side * n_experts; i += blockDim.x) {
            const uint32_t e = i % n_experts;
            uint32_t b = 0, t = 0;
#pragma unroll 8
            for (uint32_t c = i / n_experts; c < gridDim.x; c += side) {
                const uint32_t h = hist[(uint64_t)c * n_experts + e];
                t += h;
                if (c < blockIdx.x) b += h;
            }
            atomicAdd(&before[e], b);
            atomicAdd(&total[e], t);
        }
    }
    __syncthreads();
    if (!hist) {
        for (uint32_t e = threadIdx.x; e < n_experts; e += blockDim.x) {
            uint32_t t = 0;
            for (int w = 0; w < kLayoutWarps; ++w) t += layout_smem[w * n_experts + e];
            total[e] = t;
        }
        __syncthreads();
    }
    if (warp == 0) {
        uint32_t run = 0;
        for (uint32_t e0 = 0; e0 < n_experts; e0 += 32) {
            const uint32_t e = e0 + lane;
            const uint32_t v = e < n_experts ? (total[e] + kFp8Block - 1) / kFp8Block * kFp8Block : 0;
            uint32_t s = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(~0u, s, d);
                if (lane >= d) s += o;
            }
            if (e < n_experts) first[e] = run + s - v;
            run += __shfl_sync(~0u, s, 31);
        }
        if (lane == 0) first[n_experts] = run;
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < n_experts; e += blockDim.x) {
        uint32_t run = first[e] + before[e];
        for (int w = 0; w < kLayoutWarps; ++w) {
            const uint32_t v = layout_smem[w * n_experts + e];
            layout_smem[w * n_experts + e] = run;
            run += v;
        }
    }
    // the rows that fill the segments up, and the outputs per expert, spread over the blocks
    for (uint32_t e = blockIdx.x * kLayoutWarps + warp; e < n_experts; e += gridDim.x * kLayoutWarps) {
        for (uint32_t r = first[e] + total[e] + lane; r < first[e + 1]; r += 32) slot_of_row[r] = -1;
        if (lane == 0) starts[e] = (int32_t)first[e], counts[e] = (int32_t)total[e];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) starts[n_experts] = (int32_t)first[n_experts];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kLayoutRounds; ++r) {
        const uint64_t i = base + r * 32 + lane;
        const uint32_t peers = __match_any_sync(~0u, ids[r]);
        const bool some = ids[r] < n_experts;
        uint32_t row = 0;
        if (some) row = next[ids[r]] + __popc(peers & ((1u << lane) - 1));
        __syncwarp();
        if (some && lane == __ffs(peers) - 1) next[ids[r]] += __popc(peers);
        __syncwarp();
        if (i < n_slots) {
            row_of_slot[i] = some ? (int32_t)row : -1;
            if (some) slot_of_row[row] = (int32_t)i;
        }
    }
}

// ------------------------------------------------------------------------------------------ weighted sum
// A thread has N neighbouring columns of one token and adds its rows' up in fp32; a row is
// read once, so the kernel is bound by memory.  (Index: uint32_t wherever it holds every thread's number: a division of 64 bits
// costs as much as all the rest.)

constexpr int kCombineThreads = 256;

template <int DT, int N, class Index>
__global__ void __launch_bounds__(kCombineThreads)
    combine_kernel(const value_t<DT>* __restrict__ rows, uint32_t n_rows, uint64_t rows_stride,
                   const int32_t* __restrict__ row_of_slot, const float* __restrict__ weights, Index n, uint32_t per,
                   uint32_t top_k, value_t<DT>* __restrict__ out, uint64_t out_stride) {
    pdl_wait();
    const Index step = (Index)gridDim.x * blockDim.x;
    for (Index i = (Index)blockIdx.x * blockDim.x + threadIdx.x; i < n;) {
        const Index t = i / per;
        const uint32_t c = (uint32_t)(i - t * per) * N;
        const int32_t* at = row_of_slot + (uint64_t)t * top_k;
        const float* w = weights ? weights + (uint64_t)t * top_k : nullptr;
        float sum[N] = {};
#pragma unroll 4
        for (uint32_t j = 0; j < top_k; ++j) {
            const uint32_t row = (uint32_t)at[j];
            if (row >= n_rows) continue;
            const float scale = w ? w[j] : 1.f;
            float v[N];
            load_values<DT, N>(rows + row * rows_stride + c, v);
#pragma unroll
            for (int q = 0; q < N; ++q) sum[q] = fmaf(scale, v[q], sum[q]);
        }
        store_values<DT, N>(out + t * out_stride + c, sum);
        if (n - i <= step) break;  // (i + step may not fit)
        i += step;
    }
}

// A warp per slot: the dot product of the token's gradient with the slot's row, and the row's gradient.
template <int DT, int N>
__global__ void __launch_bounds__(kCombineThreads)
    combine_backward_kernel(const value_t<DT>* __restrict__ dout, uint64_t dout_stride, const value_t<DT>* __restrict__ rows,
                            uint32_t n_rows, uint64_t rows_stride, const int32_t* __restrict__ row_of_slot,
                            const float* __restrict__ weights, uint64_t n_slots, uint32_t top_k, uint32_t cols,
                            float* __restrict__ dweights, value_t<DT>* __restrict__ drows, uint64_t drows_stride) {
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const uint64_t warps = (uint64_t)gridDim.x * (kCombineThreads / 32);
    for (uint64_t i = (uint64_t)blockIdx.x * (kCombineThreads / 32) + (threadIdx.x >> 5); i < n_slots; i += warps) {
        const uint32_t row = (uint32_t)row_of_slot[i];
        float dot = 0.f;
        if (row < n_rows) {
            const float w = weights ? weights[i] : 1.f;
            const value_t<DT>* d = dout + i / top_k * dout_stride;
            const value_t<DT>* r = rows + row * rows_stride;
#pragma unroll 4
            for (uint32_t c = lane * N; c < cols; c += 32 * N) {
                float dv[N], rv[N];
                load_values<DT, N>(d + c, dv);
                load_values<DT, N>(r + c, rv);
#pragma unroll
                for (int q = 0; q < N; ++q) dot = fmaf(dv[q], rv[q], dot);
                if (drows) {
#pragma unroll
                    for (int q = 0; q < N; ++q) dv[q] *= w;
                    store_values<DT, N>(drows + row * drows_stride + c, dv);
                }
            }
        }
#pragma unroll
        for (int s = 16; s; s >>= 1) dot += __shfl_xor_sync(~0u, dot, s);
        if (lane == 0) dweights[i] = dot;
    }
}

// f(N as a constant): the most neighbouring values that one access can take at all of these addresses and strides
template <int DT, class F>
static void with_width(uint64_t bits, F&& f) {
    constexpr uint64_t v = sizeof(value_t<DT>);
    if (!(bits & 15)) f(std::integral_constant<int, 16 / v>());
    else if (!(bits & (4 * v - 1))) f(std::integral_constant<int, 4>());
    else if (!(bits & (2 * v - 1))) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 1>());
}

static uint32_t blocks_for(uint64_t work, uint64_t per_block) {
    const uint64_t b = (work + per_block - 1) / per_block;
    return (uint32_t)(b < 148ull * 64 ? (b ? b : 1) : 148ull * 64);
}

}  // namespace ciera

using namespace ciera;

extern "C" uint64_t ciera_expert_rows_capacity(uint64_t n_slots, uint32_t n_experts) {
    return kFp8Block * (n_slots / kFp8Block + (n_slots < n_experts ? n_slots : n_experts));
}

static uint64_t layout_chunks(uint64_t n_slots) { return (n_slots + kLayoutChunk - 1) / kLayoutChunk; }

extern "C" size_t ciera_expert_layout_workspace_bytes(uint64_t n_slots, uint32_t n_experts) {
    const uint64_t chunks = layout_chunks(n_slots);
    return chunks > 1 ? (size_t)((chunks + (chunks >= kLayoutScanFrom)) * n_experts * sizeof(uint32_t)) : 16;
}

extern "C" int ciera_expert_layout(const int32_t* experts_dev, uint64_t n_slots, uint32_t n_experts, int32_t* starts_dev,
                                   int32_t* counts_dev, int32_t* row_of_slot_dev, int32_t* slot_of_row_dev, void* workspace,
                                   void* stream) {
    if (n_experts < 1 || n_experts > kMaxExperts || n_slots > (1ull << 30) || !starts_dev || !counts_dev ||
        (n_slots && (!experts_dev || !row_of_slot_dev || !slot_of_row_dev || !workspace)))
        return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(experts_dev, 4) || !aligned_to(starts_dev, 4) || !aligned_to(counts_dev, 4) ||
        !aligned_to(row_of_slot_dev, 4) || !aligned_to(slot_of_row_dev, 4) || !aligned_to(workspace, 4))
        return CIERA_ERR_MISALIGNED;
    const uint64_t chunks = layout_chunks(n_slots);
    const cudaStream_t s = (cudaStream_t)stream;
    const uint32_t* hist = nullptr;
    const bool scanned = chunks >= kLayoutScanFrom;
    const auto place = scanned ? layout_place<true> : layout_place<false>;
    const auto place_bytes = [](uint32_t experts) { return sizeof(uint32_t) * ((kLayoutWarps + 3) * experts + 1); };  // up to 78 KB
    const size_t smem = place_bytes(n_experts);
    cudaError_t e = cudaSuccess;
    if (smem > 48 * 1024) {  // (always the same limit: another host thread's call must not lower it before this launch)
        e = cudaFuncSetAttribute(place, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)place_bytes(kMaxExperts));
        if (e != cudaSuccess) return record_cuda_error(e);
    }
    if (chunks > 1) {
        e = launch_after(layout_count, dim3((uint32_t)chunks), kLayoutWarps * 32, sizeof(uint32_t) * n_experts, s, experts_dev, n_slots,
                         n_experts, (uint32_t*)workspace);
        if (e != cudaSuccess) return record_cuda_error(e);
        count_launch();
        hist = (const uint32_t*)workspace;
    }
    if (scanned) {
        e = launch_after(layout_scan, dim3((n_experts + 31) / 32), kScanStretches * 32, 0, s, (uint32_t*)workspace, (uint32_t)chunks, n_experts);
        if (e != cudaSuccess) return record_cuda_error(e);
        count_launch();
    }
    e = launch_after(place, dim3((uint32_t)(chunks ? chunks : 1)), kLayoutWarps * 32, smem, s, experts_dev, n_slots, n_experts, hist,
                     starts_dev, counts_dev, row_of_slot_dev, slot_of_row_dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}

static int combine_check(int dtype, uint64_t n_rows, uint64_t rows_stride, const void* rows, const int32_t* at,
                         const float* weights, uint64_t n_tokens, uint32_t top_k, uint64_t cols, const void* out,
                         uint64_t out_stride) {
    if (top_k < 1 || top_k > 32 || cols < 1 || cols > kMaxExtent || n_tokens > kMaxExtent / top_k || n_rows > kMaxExtent ||
        (n_rows > 1 && rows_stride < cols) || (n_tokens > 1 && out_stride < cols) || (n_rows && !rows))
        return CIERA_ERR_INVALID_ARG;
    if (n_tokens && (!at || !out)) return CIERA_ERR_INVALID_ARG;
    if (dtype != CIERA_BF16 && dtype != CIERA_FP32 && dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(rows, dtype_bytes(dtype)) || !aligned_to(out, dtype_bytes(dtype)) || !aligned_to(at, 4) ||
        !aligned_to(weights, 4))
        return CIERA_ERR_MISALIGNED;
    return CIERA_OK;
}

extern "C" int ciera_expert_combine(int dtype, const void* rows_dev, uint64_t n_rows, uint64_t rows_stride,
                                    const int32_t* row_of_slot_dev, const float* weights_dev, uint64_t n_tokens,
                                    uint32_t top_k, uint64_t cols, void* out_dev, uint64_t out_stride, void* stream) {
    const int rc = combine_check(dtype, n_rows, rows_stride, rows_dev, row_of_slot_dev, weights_dev, n_tokens, top_k, cols,
                                 out_dev, out_stride);
    if (rc || !n_tokens) return rc;
    cudaError_t e = cudaSuccess;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const uint64_t v = dtype_bytes(DT);
        const uint64_t bits = (uint64_t)rows_dev | (uint64_t)out_dev | rows_stride * v | out_stride * v | cols * v;
        with_width<DT>(bits, [&](auto width) {
            constexpr int N = decltype(width)::value;
            const uint32_t per = (uint32_t)((cols + N - 1) / N);
            const uint64_t n = n_tokens * per;
            const auto go = [&](auto index) {
                using Index = decltype(index);
                e = launch_after(combine_kernel<DT, N, Index>, dim3(blocks_for(n, kCombineThreads)), kCombineThreads, 0, (cudaStream_t)stream,
                                 (const value_t<DT>*)rows_dev, (uint32_t)n_rows, rows_stride, row_of_slot_dev, weights_dev, (Index)n, per,
                                 top_k, (value_t<DT>*)out_dev, out_stride);
            };
            n >> 32 ? go(uint64_t()) : go(uint32_t());
        });
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}

extern "C" int ciera_expert_combine_backward(int dtype, const void* dout_dev, uint64_t dout_stride, const void* rows_dev,
                                             uint64_t n_rows, uint64_t rows_stride, const int32_t* row_of_slot_dev,
                                             const float* weights_dev, uint64_t n_tokens, uint32_t top_k, uint64_t cols,
                                             float* dweights_dev, void* drows_dev, uint64_t drows_stride, void* stream) {
    const int rc = combine_check(dtype, n_rows, rows_stride, rows_dev, row_of_slot_dev, weights_dev, n_tokens, top_k, cols,
                                 dout_dev, dout_stride);
    if (rc) return rc;
    if ((n_tokens && !dweights_dev) || (drows_dev && n_rows > 1 && drows_stride < cols)) return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(dweights_dev, 4) || !aligned_to(drows_dev, dtype_bytes(dtype))) return CIERA_ERR_MISALIGNED;
    if (!n_tokens) return CIERA_OK;
    cudaError_t e = cudaSuccess;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const uint64_t v = dtype_bytes(DT);
        const uint64_t bits = (uint64_t)rows_dev | (uint64_t)dout_dev | (uint64_t)drows_dev | rows_stride * v |
                              dout_stride * v | (drows_dev ? drows_stride * v : 0) | cols * v;
        with_width<DT>(bits, [&](auto width) {
            constexpr int N = decltype(width)::value;
            e = launch_after(combine_backward_kernel<DT, N>, dim3(blocks_for(n_tokens * top_k, kCombineThreads / 32)),
                             kCombineThreads, 0, (cudaStream_t)stream, (const value_t<DT>*)dout_dev, dout_stride,
                             (const value_t<DT>*)rows_dev, (uint32_t)n_rows, rows_stride, row_of_slot_dev, weights_dev,
                             n_tokens * top_k, top_k, (uint32_t)cols, dweights_dev, (value_t<DT>*)drows_dev, drows_stride);
        });
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
