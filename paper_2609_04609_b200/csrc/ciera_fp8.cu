// Operands of the 8-bit products: rows or matrices rounded to e4m3 with a power of two for each 128 values.
//
// A block of threads has a tile of 128 x 128 values.  A warp has 16 rows, a lane 4 neighbouring columns of each, so a row's
// largest magnitude is one reduction over the warp and the tile is read and kept in registers once for both orientations;
// the transposed copy goes through shared memory to be written 128 bytes at a time.  Memory bounds it.
#include <type_traits>

#include "ciera_numeric.cuh"

namespace ciera {

constexpr int kTileThreads = 256;
constexpr int kTileRows = 16;  // rows of a warp
constexpr int kTransposedPitch = 128 + 16;

struct RowsArgs {
    uint64_t x_stride, grad_stride, q_stride, scales_stride, qt_stride, scales_t_stride;
    uint64_t x_rows;
    const int32_t* slot_of_row;
    const float* row_weights;
    const int32_t* starts;
    uint32_t rows, cols, top_k, n_experts;
    uint8_t* q;
    uint8_t* scales;
    uint8_t* qt;
    uint8_t* scales_t;
};

// The scale byte of a block whose largest magnitude has these bits: the least s >= -126 with amax <= 1.75 * 2^8 * 2^s.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax >= 0x7f800000u) return 255u;
    if (amax == 0u) return 127u;
    const int s = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(max(s, -126) + 127);
}
// 2^-s; NaN for byte 255, so that every value of the block becomes one
__device__ __forceinline__ float inverse_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : (254u - byte) << 23);
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d, float inv) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}

__device__ __forceinline__ float sigmoid32(float g) { return 1.f / (1.f + expf(-g)); }

// One value of the rows: x's, silu(g) * u, or one of their gradients.
template <int DT, int SRC>
__device__ __forceinline__ float source_value(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c,
                                              uint32_t cols) {
    if constexpr (SRC == CIERA_SOURCE_ROWS) {
        return ValueOf<DT>::get(x[c]);
    } else if constexpr (SRC == CIERA_SOURCE_SWIGLU) {
        const float g = ValueOf<DT>::get(x[c]), u = ValueOf<DT>::get(x[cols + c]);
        return g * sigmoid32(g) * u;
    } else {
        const uint32_t f = cols / 2, j = c < f ? c : c - f;
        const float g = ValueOf<DT>::get(x[j]), u = ValueOf<DT>::get(x[f + j]), d = ValueOf<DT>::get(grad[j]);
        const float s = sigmoid32(g);
        return c < f ? d * u * s * (1.f + g * (1.f - s)) : d * g * s;
    }
}

// the same in 64 bits, its magnitude
template <int DT, int SRC>
__device__ double source_magnitude(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c, uint32_t cols) {
    const uint32_t f = SRC == CIERA_SOURCE_SWIGLU ? cols : cols / 2, j = c < f ? c : c - f;
    const double g = ValueOf<DT>::get(x[j]), u = ValueOf<DT>::get(x[f + j]);
    const double s = 1.0 / (1.0 + exp(-g));
    if constexpr (SRC == CIERA_SOURCE_SWIGLU) {
        return fabs(g * s * u);
    } else {
        const double d = ValueOf<DT>::get(grad[j]);
        return fabs(c < f ? d * u * s * (1.0 + g * (1.0 - s)) : d * g * s);
    }
}

// A largest magnitude so close above or below 1.75 * 2^n that 32 bits do not say on which side it is: the values behind
// an exponential are off by less than 2^-20 of themselves.
__device__ __forceinline__ bool at_border(uint32_t amax) {
    return amax < 0x7f800000u && amax > 0u && (uint32_t)((amax & 0x7fffffu) - 0x600000u + 16u) <= 32u;
}
// amax by its value in 64 bits: on the side of the border on which that is
__device__ __forceinline__ uint32_t settle(uint32_t amax, double exact) {
    const uint32_t border = (amax & 0x7f800000u) | 0x600000u;
    return exact > (double)__uint_as_float(border) ? border + 1u : border;
}

template <int DT, int SRC, bool T>
__global__ void __launch_bounds__(kTileThreads) quantize_rows_kernel(const RowsArgs a, const value_t<DT>* __restrict__ x,
                                                                     const value_t<DT>* __restrict__ grad) {
    __shared__ uint32_t col_max[T ? kTileThreads / 32 : 1][128];
    __shared__ __align__(16) uint8_t turned[T ? 128 * kTransposedPitch : 16];
    pdl_wait();
    const uint32_t row0 = blockIdx.x * 128u, col0 = blockIdx.y * 128u;
    const uint32_t rows = a.starts ? min((uint32_t)max(a.starts[a.n_experts], 0), a.rows) : a.rows;
    if (row0 >= rows) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c0 = col0 + lane * 4;
    float v[kTileRows][4];
    const value_t<DT>* xr[kTileRows];
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        const uint32_t r = row0 + warp * kTileRows + i;
        uint64_t from = r;
        float w = 1.f;
        bool some = r < rows;
        if (some && a.slot_of_row) {
            const int32_t slot = a.slot_of_row[r];
            some = slot >= 0 && (uint64_t)slot < a.x_rows * a.top_k;
            if (SRC == CIERA_SOURCE_ROWS) from = (uint32_t)max(slot, 0) / a.top_k;
            if (some && a.row_weights) w = a.row_weights[slot];
        } else if (some) {
            some = r < a.x_rows;
        }
        xr[i] = some ? x + from * a.x_stride : nullptr;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[i][j] = 0.f;
            if (some && c0 + j < a.cols) {
                v[i][j] = source_value<DT, SRC>(xr[i], SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + from * a.grad_stride : nullptr,
                                                c0 + j, a.cols);
                if (SRC == CIERA_SOURCE_ROWS && a.row_weights) v[i][j] *= w;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        const uint32_t r = row0 + warp * kTileRows + i;
        uint32_t amax = max(max(magnitude(v[i][0]), magnitude(v[i][1])), max(magnitude(v[i][2]), magnitude(v[i][3])));
        amax = __reduce_max_sync(~0u, amax);
        if constexpr (SRC != CIERA_SOURCE_ROWS) {
            if (at_border(amax)) {
                double m = 0.0;
                for (int j = 0; j < 4; ++j)
                    if (xr[i] && c0 + j < a.cols)
                        m = fmax(m, source_magnitude<DT, SRC>(xr[i], SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + (uint64_t)r * a.grad_stride : nullptr,
                                                              c0 + j, a.cols));
#pragma unroll
                for (int d = 16; d; d >>= 1) m = fmax(m, __shfl_xor_sync(~0u, m, d));
                amax = settle(amax, m);
            }
        }
        const uint32_t byte = scale_byte(amax);
        if (r >= rows) continue;
        if (lane == 0) a.scales[(uint64_t)blockIdx.y * a.scales_stride + r] = (uint8_t)byte;
        const uint32_t q = to_e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3], inverse_scale(byte));
        uint8_t* to = a.q + (uint64_t)r * a.q_stride + c0;
        if (c0 + 3 < a.cols) {
            *reinterpret_cast<uint32_t*>(to) = q;
        } else {
            for (int j = 0; j < 3; ++j)
                if (c0 + j < a.cols) to[j] = (uint8_t)(q >> (8 * j));
        }
    }
    if constexpr (T) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kTileRows; ++i) m = max(m, magnitude(v[i][j]));
            col_max[warp][lane * 4 + j] = m;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t c = c0 + j;
            uint32_t amax = 0;
#pragma unroll
            for (int w = 0; w < kTileThreads / 32; ++w) amax = max(amax, col_max[w][lane * 4 + j]);
            if constexpr (SRC != CIERA_SOURCE_ROWS) {
                if (at_border(amax)) {  // (the same in every warp; each goes over the whole column)
                    double m = 0.0;
                    for (uint32_t r = row0; r < min(row0 + 128u, rows) && c < a.cols; ++r) {
                        if (a.slot_of_row) {
                            const int32_t slot = a.slot_of_row[r];
                            if (slot < 0 || (uint64_t)slot >= a.x_rows * a.top_k) continue;
                        } else if (r >= a.x_rows) continue;
                        m = fmax(m, source_magnitude<DT, SRC>(x + (uint64_t)r * a.x_stride,
                                                              SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + (uint64_t)r * a.grad_stride : nullptr, c, a.cols));
                    }
                    amax = settle(amax, m);
                }
            }
            const uint32_t byte = scale_byte(amax);
            const float inv = inverse_scale(byte);
            if (warp == 0 && c < a.cols) a.scales_t[(uint64_t)blockIdx.x * a.scales_t_stride + c] = (uint8_t)byte;
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = to_e4m3x4(v[4 * i][j], v[4 * i + 1][j], v[4 * i + 2][j], v[4 * i + 3][j], inv);
            *reinterpret_cast<uint4*>(turned + (lane * 4 + j) * kTransposedPitch + warp * kTileRows) = make_uint4(q[0], q[1], q[2], q[3]);
        }
        __syncthreads();
        for (int k = threadIdx.x; k < 128 * 8; k += kTileThreads) {
            const uint32_t c = col0 + (k >> 3), r = row0 + (k & 7) * 16;
            if (c >= a.cols || r >= rows) continue;
            const uint4 q = *reinterpret_cast<const uint4*>(turned + (k >> 3) * kTransposedPitch + (k & 7) * 16);
            uint8_t* to = a.qt + (uint64_t)c * a.qt_stride + r;
            if (r + 15 < rows) {
                *reinterpret_cast<uint4*>(to) = q;
            } else {
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                for (uint32_t i = 0; r + i < rows; ++i) to[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
}

struct BlocksArgs {
    uint64_t x_stride, x_matrix_stride, q_stride, q_matrix_stride, scales_stride, scales_matrix_stride;
    uint64_t qt_stride, qt_matrix_stride, scales_t_stride, scales_t_matrix_stride;
    uint32_t rows, cols, row_blocks, col_blocks;
    uint8_t* q;
    uint8_t* scales;
    uint8_t* qt;
    uint8_t* scales_t;
};

template <int DT, bool T>
__global__ void __launch_bounds__(kTileThreads) quantize_blocks_kernel(const BlocksArgs a, const value_t<DT>* __restrict__ x) {
    __shared__ uint32_t warp_max[kTileThreads / 32];
    __shared__ __align__(16) uint8_t turned[T ? 128 * kTransposedPitch : 16];
    pdl_wait();
    const uint32_t matrix = blockIdx.x / a.row_blocks, rb = blockIdx.x % a.row_blocks;
    const uint32_t row0 = rb * 128u, col0 = blockIdx.y * 128u;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c0 = col0 + lane * 4;
    float v[kTileRows][4];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        const uint32_t r = row0 + warp * kTileRows + i;
        const value_t<DT>* xr = x + matrix * a.x_matrix_stride + r * a.x_stride;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[i][j] = r < a.rows && c0 + j < a.cols ? ValueOf<DT>::get(xr[c0 + j]) : 0.f;
            amax = max(amax, magnitude(v[i][j]));
        }
    }
    amax = __reduce_max_sync(~0u, amax);
    if (lane == 0) warp_max[warp] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTileThreads / 32; ++w) amax = max(amax, warp_max[w]);
    const uint32_t byte = scale_byte(amax);
    const float inv = inverse_scale(byte);
    if (threadIdx.x == 0) {
        a.scales[matrix * a.scales_matrix_stride + rb * a.scales_stride + blockIdx.y] = (uint8_t)byte;
        if (T) a.scales_t[matrix * a.scales_t_matrix_stride + blockIdx.y * a.scales_t_stride + rb] = (uint8_t)byte;
    }
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        const uint32_t r = row0 + warp * kTileRows + i;
        if (r >= a.rows) break;
        const uint32_t q = to_e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3], inv);
        uint8_t* to = a.q + matrix * a.q_matrix_stride + r * a.q_stride + c0;
        if (c0 + 3 < a.cols) {
            *reinterpret_cast<uint32_t*>(to) = q;
        } else {
            for (int j = 0; j < 3; ++j)
                if (c0 + j < a.cols) to[j] = (uint8_t)(q >> (8 * j));
        }
    }
    if constexpr (T) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = to_e4m3x4(v[4 * i][j], v[4 * i + 1][j], v[4 * i + 2][j], v[4 * i + 3][j], inv);
            *reinterpret_cast<uint4*>(turned + (lane * 4 + j) * kTransposedPitch + warp * kTileRows) = make_uint4(q[0], q[1], q[2], q[3]);
        }
        __syncthreads();
        for (int k = threadIdx.x; k < 128 * 8; k += kTileThreads) {
            const uint32_t c = col0 + (k >> 3), r = row0 + (k & 7) * 16;
            if (c >= a.cols || r >= a.rows) continue;
            const uint4 q = *reinterpret_cast<const uint4*>(turned + (k >> 3) * kTransposedPitch + (k & 7) * 16);
            uint8_t* to = a.qt + matrix * a.qt_matrix_stride + c * a.qt_stride + r;
            if (r + 15 < a.rows) {
                *reinterpret_cast<uint4*>(to) = q;
            } else {
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                for (uint32_t i = 0; r + i < a.rows; ++i) to[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
}

// (the stride of a single row counts for nothing)
static bool fp8_tensor_ok(const void* p, uint64_t rows, uint64_t stride) { return aligned_to(p, 16) && (rows <= 1 || !(stride & 15)); }

}  // namespace ciera

using namespace ciera;

extern "C" int ciera_fp8_quantize_rows(const ciera_fp8_rows* p, void* stream) {
    if (!p || p->rows > kMaxExtent || p->cols > kMaxExtent || p->x_rows > kMaxExtent) return CIERA_ERR_INVALID_ARG;
    const int src = p->source;
    if (src != CIERA_SOURCE_ROWS && src != CIERA_SOURCE_SWIGLU && src != CIERA_SOURCE_SWIGLU_BACKWARD) return CIERA_ERR_INVALID_ARG;
    if (p->dtype != CIERA_BF16 && p->dtype != CIERA_FP32 && p->dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if (!p->rows) return CIERA_OK;
    const bool back = src == CIERA_SOURCE_SWIGLU_BACKWARD, turned = p->qt != nullptr;
    const uint64_t width = src == CIERA_SOURCE_SWIGLU ? 2 * p->cols : p->cols;
    if (p->cols < 1 || (p->x_rows && !p->x) || !p->q || !p->scales || turned != (p->scales_t != nullptr) ||
        back != (p->grad != nullptr) || (back && (p->cols & 1)) || (p->row_weights && (src != CIERA_SOURCE_ROWS || !p->slot_of_row)) ||
        (p->x_rows > 1 && p->x_stride < width) || (back && p->x_rows > 1 && p->grad_stride < p->cols / 2) ||
        (p->rows > 1 && p->q_stride < p->cols) || p->scales_stride < p->rows || (turned && (p->scales_t_stride < p->cols)) ||
        (turned && p->cols > 1 && p->qt_stride < p->rows) || (p->slot_of_row && (p->top_k < 1 || p->top_k > 32)) ||
        (p->slot_of_row && p->x_rows * p->top_k > kMaxExtent) || (p->starts && (p->n_experts < 1 || p->n_experts > 1024)))
        return CIERA_ERR_INVALID_ARG;
    if (src != CIERA_SOURCE_ROWS && p->x_rows < p->rows) return CIERA_ERR_INVALID_ARG;
    if (!p->slot_of_row && p->x_rows < p->rows) return CIERA_ERR_INVALID_ARG;
    if (!fp8_tensor_ok(p->q, p->rows, p->q_stride) || (turned && !fp8_tensor_ok(p->qt, p->cols, p->qt_stride)) || !aligned_to(p->x, dtype_bytes(p->dtype)) ||
        !aligned_to(p->grad, dtype_bytes(p->dtype)) || !aligned_to(p->slot_of_row, 4) || !aligned_to(p->row_weights, 4) ||
        !aligned_to(p->starts, 4))
        return CIERA_ERR_MISALIGNED;
    if ((p->cols + 127) / 128 > 65535) return CIERA_ERR_UNSUPPORTED;
    const RowsArgs a{p->x_stride, p->grad_stride, p->q_stride, p->scales_stride, p->qt_stride, p->scales_t_stride, p->x_rows,
                     p->slot_of_row, p->row_weights, p->starts, (uint32_t)p->rows, (uint32_t)p->cols,
                     p->slot_of_row ? p->top_k : 1u, p->n_experts, (uint8_t*)p->q, p->scales, (uint8_t*)p->qt, p->scales_t};
    const dim3 grid((uint32_t)((p->rows + 127) / 128), (uint32_t)((p->cols + 127) / 128));
    cudaError_t e = cudaSuccess;
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto kernel) {
            e = launch_after(kernel, grid, kTileThreads, 0, (cudaStream_t)stream, a, (const value_t<DT>*)p->x, (const value_t<DT>*)p->grad);
        };
        if (src == CIERA_SOURCE_ROWS) turned ? go(quantize_rows_kernel<DT, CIERA_SOURCE_ROWS, true>) : go(quantize_rows_kernel<DT, CIERA_SOURCE_ROWS, false>);
        else if (!back) turned ? go(quantize_rows_kernel<DT, CIERA_SOURCE_SWIGLU, true>) : go(quantize_rows_kernel<DT, CIERA_SOURCE_SWIGLU, false>);
        else turned ? go(quantize_rows_kernel<DT, CIERA_SOURCE_SWIGLU_BACKWARD, true>) : go(quantize_rows_kernel<DT, CIERA_SOURCE_SWIGLU_BACKWARD, false>);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}

extern "C" int ciera_fp8_quantize_blocks(const ciera_fp8_blocks* p, void* stream) {
    if (!p || p->rows > kMaxExtent || p->cols > kMaxExtent) return CIERA_ERR_INVALID_ARG;
    if (p->dtype != CIERA_BF16 && p->dtype != CIERA_FP32 && p->dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if (!p->matrices) return CIERA_OK;
    const bool turned = p->qt != nullptr;
    const uint64_t rb = (p->rows + 127) / 128, cb = (p->cols + 127) / 128;
    if (p->rows < 1 || p->cols < 1 || !p->x || !p->q || !p->scales || turned != (p->scales_t != nullptr) ||
        (p->rows > 1 && (p->x_stride < p->cols || p->q_stride < p->cols)) || (rb > 1 && p->scales_stride < cb) ||
        (turned && ((p->cols > 1 && p->qt_stride < p->rows) || (cb > 1 && p->scales_t_stride < rb))))
        return CIERA_ERR_INVALID_ARG;
    const bool several = p->matrices > 1;
    if (!fp8_tensor_ok(p->q, p->rows, p->q_stride) || (several && (p->q_matrix_stride & 15)) ||
        (turned && (!fp8_tensor_ok(p->qt, p->cols, p->qt_stride) || (several && (p->qt_matrix_stride & 15)))) ||
        !aligned_to(p->x, dtype_bytes(p->dtype)))
        return CIERA_ERR_MISALIGNED;
    if (cb > 65535 || rb * p->matrices > kMaxExtent) return CIERA_ERR_UNSUPPORTED;
    const BlocksArgs a{p->x_stride, p->x_matrix_stride, p->q_stride, p->q_matrix_stride, p->scales_stride, p->scales_matrix_stride,
                       p->qt_stride, p->qt_matrix_stride, p->scales_t_stride, p->scales_t_matrix_stride,
                       (uint32_t)p->rows, (uint32_t)p->cols, (uint32_t)rb, (uint32_t)cb, (uint8_t*)p->q, p->scales, (uint8_t*)p->qt, p->scales_t};
    const dim3 grid((uint32_t)(rb * p->matrices), (uint32_t)cb);
    cudaError_t e = cudaSuccess;
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto kernel) { e = launch_after(kernel, grid, kTileThreads, 0, (cudaStream_t)stream, a, (const value_t<DT>*)p->x); };
        turned ? go(quantize_blocks_kernel<DT, true>) : go(quantize_blocks_kernel<DT, false>);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
