// Products of e4m3 operands with a power of two for each block of 128 values.
//
// A first form on the ordinary cores: a block of threads has 64 x 64 results, dequantises 32 values of the contraction at a
// time into shared memory and adds up in fp32.
#include <type_traits>

#include "ciera_numeric.cuh"

namespace ciera {

struct ProductArgs {
    uint64_t a_stride, a_scales_stride, b_stride, b_matrix_stride, b_scales_stride, b_scales_matrix_stride;
    uint64_t out_stride, out_matrix_stride;
    const uint8_t* a;
    const uint8_t* a_scales;
    const uint8_t* b;
    const uint8_t* b_scales;
    const int32_t* starts;
    int32_t* status;
    uint32_t m, n, k, n_experts;
    int32_t b_blocks;
};

__device__ __forceinline__ float from_e4m3(uint8_t v) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)));
}
__device__ __forceinline__ float scale_of(uint8_t byte) {
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : (uint32_t)byte << 23);
}

// grid: columns of out, rows of out, experts
template <int MODE, int DT>
__global__ void __launch_bounds__(256) product_kernel(const ProductArgs p, value_t<DT>* __restrict__ out) {
    __shared__ float sa[32][65], sb[32][65];
    pdl_wait();
    const uint32_t e = blockIdx.z;
    uint32_t lo = 0, hi = MODE == CIERA_PRODUCT_CONTRACT ? p.k : p.m;
    if (MODE != CIERA_PRODUCT_DENSE) {
        const uint32_t most = hi;
        bool bad = p.starts[0] != 0;
        for (uint32_t i = threadIdx.x; i < p.n_experts; i += blockDim.x)
            bad |= p.starts[i] > p.starts[i + 1] || (p.starts[i + 1] & 127) || (uint32_t)p.starts[i + 1] > most;
        if (__syncthreads_or(bad)) {
            if (p.status && threadIdx.x == 0) atomicCAS(p.status, 0, (int32_t)CIERA_ERR_CORRUPT);
            return;
        }
        lo = p.starts[e], hi = p.starts[e + 1];
    }
    const uint32_t m0 = (MODE == CIERA_PRODUCT_ROWS ? lo : 0) + blockIdx.y * 64, n0 = blockIdx.x * 64;
    const uint32_t m1 = MODE == CIERA_PRODUCT_ROWS ? hi : p.m;
    const uint32_t k0 = MODE == CIERA_PRODUCT_CONTRACT ? lo : 0, k1 = MODE == CIERA_PRODUCT_CONTRACT ? hi : p.k;
    if (m0 >= m1) return;
    const uint64_t matrix = MODE == CIERA_PRODUCT_ROWS ? e : 0;
    float acc[4][4] = {};
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (uint32_t kk = k0; kk < k1; kk += 32) {
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * 32; i += 256) {
            const uint32_t k = kk + (i & 31), m = m0 + (i >> 5), n = n0 + (i >> 5);
            float va = 0.f, vb = 0.f;
            if (k < k1 && m < m1)
                va = from_e4m3(p.a[m * p.a_stride + k]) * scale_of(p.a_scales[(uint64_t)(k >> 7) * p.a_scales_stride + m]);
            if (k < k1 && n < p.n) {
                const uint8_t s = p.b_blocks ? p.b_scales[matrix * p.b_scales_matrix_stride + (uint64_t)(n >> 7) * p.b_scales_stride + (k >> 7)]
                                             : p.b_scales[(uint64_t)(k >> 7) * p.b_scales_stride + n];
                vb = from_e4m3(p.b[matrix * p.b_matrix_stride + n * p.b_stride + k]) * scale_of(s);
            }
            sa[i & 31][i >> 5] = va;
            sb[i & 31][i >> 5] = vb;
        }
        __syncthreads();
#pragma unroll 8
        for (int k = 0; k < 32; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
    }
    value_t<DT>* o = out + (MODE == CIERA_PRODUCT_CONTRACT ? e * p.out_matrix_stride : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < m1 && n < p.n) o[m * p.out_stride + n] = ValueOf<DT>::put(acc[i][j]);
        }
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
        ((rows || contract) && (p->n_experts < 1 || p->n_experts > 1024)))
        return CIERA_ERR_INVALID_ARG;
    const uint64_t kb = (p->k + 127) / 128, nb = (p->n + 127) / 128;
    if ((p->m > 1 && p->a_stride < p->k) || (p->n > 1 && p->b_stride < p->k) || (kb > 1 && p->a_scales_stride < p->m) ||
        (p->b_blocks ? nb > 1 && p->b_scales_stride < kb : kb > 1 && p->b_scales_stride < p->n) || (p->m > 1 && p->out_stride < p->n))
        return CIERA_ERR_INVALID_ARG;
    // (strides of single rows and matrices count for nothing)
    const bool several = rows && p->n_experts > 1;
    if (!aligned_to(p->a, 16) || !aligned_to(p->b, 16) || (p->m > 1 && (p->a_stride & 15)) || (p->n > 1 && (p->b_stride & 15)) ||
        (several && (p->b_matrix_stride & 15)) ||
        !aligned_to(p->out, dtype_bytes(p->out_dtype)) || !aligned_to(p->starts, 4) || !aligned_to(p->status, 4))
        return CIERA_ERR_MISALIGNED;
    if (p->a_stride >= 1ull << 40 || p->b_stride >= 1ull << 40 || p->b_matrix_stride >= 1ull << 40) return CIERA_ERR_UNSUPPORTED;
    const ProductArgs a{p->a_stride, p->a_scales_stride, p->b_stride, p->b_matrix_stride, p->b_scales_stride, p->b_scales_matrix_stride,
                        p->out_stride, p->out_matrix_stride, (const uint8_t*)p->a, p->a_scales, (const uint8_t*)p->b, p->b_scales,
                        p->starts, p->status, (uint32_t)p->m, (uint32_t)p->n, (uint32_t)p->k, p->n_experts, p->b_blocks};
    const dim3 grid((uint32_t)((p->n + 63) / 64), (uint32_t)((p->m + 63) / 64), mode == CIERA_PRODUCT_DENSE ? 1 : p->n_experts);
    if (grid.y > 65535) return CIERA_ERR_UNSUPPORTED;
    cudaError_t e = cudaSuccess;
    with_dtype(p->out_dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto kernel) { e = launch_after(kernel, grid, 256, 0, (cudaStream_t)stream, a, (value_t<DT>*)p->out); };
        if (rows) go(product_kernel<CIERA_PRODUCT_ROWS, DT>);
        else if (contract) go(product_kernel<CIERA_PRODUCT_CONTRACT, DT>);
        else go(product_kernel<CIERA_PRODUCT_DENSE, DT>);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
