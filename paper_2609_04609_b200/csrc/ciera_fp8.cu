// Operands of the 8-bit products: rows or matrices rounded to e4m3 with a power of two for each 128 values.
//
// A block of threads has a tile of 128 x 128 values.  A warp has 8 rows, a lane 4 neighbouring columns of each, so a row's
// largest magnitude is one reduction over the warp and the tile is read and kept in registers once for both orientations;
// the transposed copy goes through shared memory to be written 128 bytes at a time.  Tiles beside each other come one behind
// the other, so that blocks that run together read and write whole rows.  Square blocks are bound by memory (64 matrices of
// 2048 x 1024 in 97 us, 0.85 of the copy rate), rows in both orientations by instructions: each value is scaled and rounded
// twice (32768 rows of 2048: gathered 59 us, of which memory needs 24; weighted 79; silu(g) * u of 1024 67; its gradient 156).
#include <type_traits>

#include "ciera_fp8.cuh"
#include "ciera_swiglu.cuh"

namespace ciera {

// 16 warps of 8 rows: 32 values a thread leave room for two blocks of 512 threads on an SM, and their loads in flight.  (8 warps
// of 16 rows, two blocks of 256: dispatch of 4096 x 8 rows of 2048 in 113 us, 64 matrices of 2048 x 1024 in 205 us.)
constexpr int kTileThreads = 512;
constexpr int kTileRows = 8;  // rows of a warp

struct RowsArgs {
    uint64_t x_stride, grad_stride, q_stride, scales_stride, qt_stride, scales_t_stride;
    uint64_t x_rows;
    const int32_t* slot_of_row;
    const float* row_weights;
    const int32_t* starts;
    uint32_t rows, cols, col_tiles, top_k, n_experts;
    uint8_t* q;
    uint8_t* scales;
    uint8_t* qt;
    uint8_t* scales_t;
};

// 2^-s; NaN for byte 255, so that every value of the block becomes one
__device__ __forceinline__ float inverse_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : (254u - byte) << 23);
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d, float4 inv) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv.x, b * inv.y), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv.z, d * inv.w), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d, float inv) {
    return to_e4m3x4(a, b, c, d, make_float4(inv, inv, inv, inv));
}

// 1 + g (1 - sigmoid(g)) is zero at one g, which is here in two parts, and cancels around it: within 1/16 it comes from its series (a
// fit of degree 3 to what the definition gives in 50 digits, off by less than 2^-21 of itself), beyond that it is off by less
// than 2^-17.
__device__ __forceinline__ float swiglu_gate32(float g, float u, float d) {
    const float2 s = sigmoid32(g);
    const float from = (g + 1.27846456f) - 1.29792825e-8f;
    const float near = from * fmaf(from, fmaf(from, -0.0488740131f, -0.108919665f), 1.f);
    return d * u * s.x * (fabsf(from) < 0.0625f ? near : fmaf(g, s.y, 1.f));
}
__device__ __forceinline__ float swiglu_up32(float g, float d) { return d * g * sigmoid32(g).x; }

// Four neighbouring values of each input that four values of a row are made from, as they are read.
template <int DT>
struct RawFour {
    Pack<value_t<DT>, 4> x, up, grad;
};
template <int DT, int SRC>
__device__ __forceinline__ void read_four(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c, uint32_t cols,
                                          RawFour<DT>& raw) {
    const auto get = [](const value_t<DT>* p) { return *reinterpret_cast<const Pack<value_t<DT>, 4>*>(p); };
    if constexpr (SRC == CIERA_SOURCE_ROWS) {
        raw.x = get(x + c);
    } else if constexpr (SRC == CIERA_SOURCE_SWIGLU) {
        raw.x = get(x + c);
        raw.up = get(x + cols + c);
    } else {  // (the four are on one side)
        const uint32_t f = cols / 2, at = c < f ? c : c - f;
        raw.x = get(x + at);
        raw.grad = get(grad + at);
        raw.up = raw.x;
        if (c < f) raw.up = get(x + f + at);
    }
}
__device__ __forceinline__ uint32_t max_two(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The largest bits of gates: of the lowest one if any is negative (or of a NaN); 16-bit types two at a time.
template <int DT>
__device__ __forceinline__ void see_gates(const Pack<value_t<DT>, 4>& g, uint32_t& lowest) {
    if constexpr (DT == CIERA_FP32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) lowest = max(lowest, __float_as_uint(g.v[j]));
    } else {
        const uint2 w = *reinterpret_cast<const uint2*>(&g);
        lowest = max_two(lowest, max_two(w.x, w.y));
    }
}
template <int DT>
__device__ __forceinline__ void see_gate(float g, uint32_t& lowest) {
    const value_t<DT> v = ValueOf<DT>::put(g);
    if constexpr (DT == CIERA_FP32) lowest = max(lowest, __float_as_uint(g));
    else lowest = max_two(lowest, *reinterpret_cast<const unsigned short*>(&v));
}
// whether one is below kLowestGate (true for some NaN too)
template <int DT>
__device__ __forceinline__ bool below_lowest(uint32_t lowest) {
    if constexpr (DT == CIERA_FP32) return lowest > __float_as_uint(kLowestGate);
    constexpr uint32_t bits = DT == CIERA_BF16 ? 0xc2aeu : 0xd570u;  // -87
    return (lowest >> 16) > bits || (lowest & 0xffffu) > bits;
}
// x's, silu(g) * u, or one of their gradients; lowest: see_gates of the gates so far
template <int DT, int SRC>
__device__ __forceinline__ void make_four(const RawFour<DT>& raw, uint32_t c, uint32_t cols, float (&v)[4], uint32_t& lowest) {
    if constexpr (SRC != CIERA_SOURCE_ROWS) see_gates<DT>(raw.x, lowest);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = ValueOf<DT>::get(raw.x.v[j]);
        if constexpr (SRC == CIERA_SOURCE_ROWS) v[j] = x;
        else if constexpr (SRC == CIERA_SOURCE_SWIGLU) v[j] = swiglu32(x, ValueOf<DT>::get(raw.up.v[j]));
        else v[j] = c < cols / 2 ? swiglu_gate32(x, ValueOf<DT>::get(raw.up.v[j]), ValueOf<DT>::get(raw.grad.v[j])) : swiglu_up32(x, ValueOf<DT>::get(raw.grad.v[j]));
    }
}
// The same value by value, for rows and widths of any kind; 0 behind the row.
template <int DT, int SRC>
__device__ __forceinline__ void source_values(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c,
                                              uint32_t cols, float (&v)[4], uint32_t& lowest) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = 0.f;
        if (c + j >= cols) continue;
        if constexpr (SRC == CIERA_SOURCE_ROWS) {
            v[j] = ValueOf<DT>::get(x[c + j]);
        } else if constexpr (SRC == CIERA_SOURCE_SWIGLU) {
            const float g = ValueOf<DT>::get(x[c + j]);
            see_gate<DT>(g, lowest);
            v[j] = swiglu32(g, ValueOf<DT>::get(x[cols + c + j]));
        } else {
            const uint32_t f = cols / 2, at = c + j < f ? c + j : c + j - f;
            const float g = ValueOf<DT>::get(x[at]), u = ValueOf<DT>::get(x[f + at]), d = ValueOf<DT>::get(grad[at]);
            see_gate<DT>(g, lowest);
            v[j] = c + j < f ? swiglu_gate32(g, u, d) : swiglu_up32(g, d);
        }
    }
}

// The same in 64 bits, one value; lowest: its gate.
template <int DT, int SRC>
__device__ double source_value64(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c, uint32_t cols, float& lowest) {
    const uint32_t f = SRC == CIERA_SOURCE_SWIGLU ? cols : cols / 2, j = c < f ? c : c - f;
    const double g = lowest = ValueOf<DT>::get(x[j]), u = ValueOf<DT>::get(x[f + j]);
    const double s = 1.0 / (1.0 + exp(-g));
    if constexpr (SRC == CIERA_SOURCE_SWIGLU) {
        return g * s * u;
    } else {
        const double d = ValueOf<DT>::get(grad[j]);
        return c < f ? d * u * s * (1.0 + g * (1.0 - s)) : d * g * s;
    }
}
template <int DT, int SRC>
__device__ __forceinline__ double source_magnitude(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c, uint32_t cols) {
    float gate;
    return fabs(source_value64<DT, SRC>(x, grad, c, cols, gate));
}

// Whether a value is zero for another reason than that it is too small for 32 bits.
template <int DT, int SRC>
__device__ __forceinline__ bool zero_factor(const value_t<DT>* __restrict__ x, const value_t<DT>* __restrict__ grad, uint32_t c, uint32_t cols) {
    const uint32_t f = SRC == CIERA_SOURCE_SWIGLU ? cols : cols / 2, j = c < f ? c : c - f;
    const float a = ValueOf<DT>::get(SRC == CIERA_SOURCE_SWIGLU ? x[j] : grad[j]);
    const float b = ValueOf<DT>::get(SRC == CIERA_SOURCE_SWIGLU || c < f ? x[f + j] : x[j]);
    return a == 0.f || b == 0.f;
}

// A largest magnitude that 32 bits do not settle: so close above or below 1.75 * 2^n that they do not say on which side it is
// (values behind an exponential are off by less than 2^-20 of themselves, the gate's gradient by less than 2^-17; 256 steps are
// 2^-15.8), or so small that a factor has left their range.
__device__ __forceinline__ bool at_border(uint32_t amax) {
    return amax < 0x7f800000u && (amax < (32u << 23) || (uint32_t)((amax & 0x7fffffu) - 0x600000u + 256u) <= 512u);
}
// the same from 64 bits, rounded up: on the side of the border on which that is
__device__ __forceinline__ uint32_t settle(double exact) { return __float_as_uint(__double2float_ru(exact)); }

// The tile's four values of each row, rounded with a scale for each row, to q.
__device__ __forceinline__ void put_four(uint8_t* to, uint32_t q, uint32_t c0, uint32_t cols) {
    if (c0 + 3 < cols) {
        *reinterpret_cast<uint32_t*>(to) = q;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (c0 + j < cols) to[j] = (uint8_t)(q >> (8 * j));
    }
}

// The bytes of rows r ... r + 15 of a transposed line, as far as there are rows.
__device__ __forceinline__ void put_sixteen(uint8_t* to, uint4 q, uint32_t r, uint32_t rows) {
    if (r + 15 < rows) {
        *reinterpret_cast<uint4*>(to) = q;
    } else {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        for (uint32_t i = 0; r + i < rows; ++i) to[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}

// Four words of four bytes, turned: byte i of word j to byte j of word i.
__device__ __forceinline__ void turn_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&t)[4]) {
    const uint32_t ab = __byte_perm(a, b, 0x5140), ab2 = __byte_perm(a, b, 0x7362);
    const uint32_t cd = __byte_perm(c, d, 0x5140), cd2 = __byte_perm(c, d, 0x7362);
    t[0] = __byte_perm(ab, cd, 0x5410);
    t[1] = __byte_perm(ab, cd, 0x7632);
    t[2] = __byte_perm(ab2, cd2, 0x5410);
    t[3] = __byte_perm(ab2, cd2, 0x7632);
}
// The 8 rounded values of warp `warp` in column 4 * lane + j go to that column's line of `turned`, 16 units of 8 bytes whose
// places are mixed by the lane, so that neither the columns of a warp nor the units of a column meet in a bank ...
__device__ __forceinline__ void turn_in(uint2* turned, int lane, int j, int warp, uint32_t lo, uint32_t hi) {
    turned[(lane * 4 + j) * 16 + (((warp >> 1) ^ (lane & 7)) << 1 | ((warp & 1) ^ (lane >> 3 & 1)))] = make_uint2(lo, hi);
}
// ... and from there to the transposed tile's rows, 16 bytes a thread.
__device__ __forceinline__ void turn_out(const uint2* turned, uint8_t* qt, uint64_t stride, uint32_t col0, uint32_t cols, uint32_t row0,
                                         uint32_t rows) {
    for (int k = threadIdx.x; k < 128 * 8; k += kTileThreads) {
        const uint32_t c = k >> 3, unit = k & 7, r = row0 + unit * 16, of = c >> 2;  // (the lane that put it there)
        if (col0 + c >= cols || r >= rows) continue;
        uint4 q = *reinterpret_cast<const uint4*>(turned + c * 16 + ((unit ^ (of & 7)) << 1));
        if (of >> 3 & 1) q = make_uint4(q.z, q.w, q.x, q.y);
        put_sixteen(qt + (uint64_t)(col0 + c) * stride + r, q, r, rows);
    }
}

template <int DT, int SRC, bool T, bool WIDE>
__global__ void __launch_bounds__(kTileThreads, 2) quantize_rows_kernel(const RowsArgs a, const value_t<DT>* __restrict__ x,
                                                                        const value_t<DT>* __restrict__ grad) {
    __shared__ __align__(16) uint32_t col_max[T ? kTileThreads / 32 : 1][128];
    __shared__ __align__(16) float col_inv[128];
    __shared__ uint32_t some_rows[T && SRC != CIERA_SOURCE_ROWS ? kTileThreads / 32 : 1];  // of a warp: those that are more than zeros
    __shared__ __align__(16) uint2 turned[T ? 128 * 16 : 2];
    pdl_wait();
    const uint32_t row_tile = blockIdx.x / a.col_tiles, col_tile = blockIdx.x - row_tile * a.col_tiles;
    const uint32_t row0 = row_tile * 128u, col0 = col_tile * 128u;
    const uint32_t rows = a.starts ? min((uint32_t)max(a.starts[a.n_experts], 0), a.rows) : a.rows;
    if (row0 >= rows) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c0 = col0 + lane * 4, first = row0 + warp * kTileRows;
    // lane i: where row i of the warp comes from
    uint32_t from = first + lane;
    float weight = 1.f;
    bool some = lane < kTileRows && from < rows;
    if (a.slot_of_row) {
        const int32_t slot = some ? a.slot_of_row[from] : -1;
        some = slot >= 0 && (uint64_t)slot < a.x_rows * a.top_k;
        if (SRC == CIERA_SOURCE_ROWS) from = (uint32_t)max(slot, 0) / a.top_k;
        if (some && a.row_weights) weight = a.row_weights[slot];
    } else {
        some = some && from < a.x_rows;
    }
    const uint32_t live = __ballot_sync(~0u, some);
    if (!some) from = 0;
    float v[kTileRows][4];
    uint32_t lowest = 0;
    if constexpr (WIDE) {
        // Rows without a slot and columns behind the row read the first of either, and are put to zero afterwards: what is read
        // stands under no condition, so that several rows' values are on their way together (one by one: silu(g) * u of
        // 32768 x 1024 in 85 us, its gradient in 178).
        constexpr int kAtOnce = SRC == CIERA_SOURCE_ROWS ? kTileRows : sizeof(value_t<DT>) == 2 ? 4 : 2;
        const bool whole = c0 < a.cols;  // (cols is a multiple of four)
        const uint32_t c = whole ? c0 : 0;
#pragma unroll
        for (int i0 = 0; i0 < kTileRows; i0 += kAtOnce) {
            RawFour<DT> raw[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const uint32_t r = __shfl_sync(~0u, from, i0 + i);
                if (a.x_rows) read_four<DT, SRC>(x + r * a.x_stride, SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + r * a.grad_stride : nullptr, c, a.cols, raw[i]);
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                make_four<DT, SRC>(raw[i], c, a.cols, v[i0 + i], lowest);
                if (!(live >> (i0 + i) & 1 && whole)) v[i0 + i][0] = v[i0 + i][1] = v[i0 + i][2] = v[i0 + i][3] = 0.f;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kTileRows; ++i) {
            const uint32_t r = __shfl_sync(~0u, from, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = 0.f;
            if (live >> i & 1 && c0 < a.cols)
                source_values<DT, SRC>(x + r * a.x_stride, SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + r * a.grad_stride : nullptr, c0, a.cols, v[i], lowest);
        }
    }
    if constexpr (SRC != CIERA_SOURCE_ROWS) {
        if (__any_sync(~0u, below_lowest<DT>(lowest))) {  // such values in 64 bits
#pragma unroll 1
            for (uint32_t n = 0; n < kTileRows * 4; ++n) {
                const uint64_t r = first + n / 4;
                const uint32_t c = c0 + n % 4;
                float gate = 0.f, value = 0.f;
                if (live >> (n / 4) & 1 && c < a.cols)
                    value = (float)source_value64<DT, SRC>(x + r * a.x_stride, SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + r * a.grad_stride : nullptr, c, a.cols, gate);
#pragma unroll
                for (int i = 0; i < kTileRows; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (n == (uint32_t)(i * 4 + j) && gate < kLowestGate) v[i][j] = value;
            }
        }
    }
    if (SRC == CIERA_SOURCE_ROWS && a.row_weights) {
#pragma unroll
        for (int i = 0; i < kTileRows; ++i) {
            const float w = __shfl_sync(~0u, weight, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] *= w;
        }
    }
    uint32_t row_max = 0;  // lane i: the largest magnitude of row i
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        uint32_t amax = max(max(magnitude(v[i][0]), magnitude(v[i][1])), max(magnitude(v[i][2]), magnitude(v[i][3])));
        amax = __reduce_max_sync(~0u, amax);
        if (lane == i) row_max = amax;
    }
    if constexpr (SRC != CIERA_SOURCE_ROWS) {
        const auto grad_row = [&](uint64_t r) { return SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + r * a.grad_stride : nullptr; };
        // Rows of zeros that stand for nothing else, tokens without a gradient among them, are looked at in 32 bits (in 64, as what
        // follows, the gradient of 32768 such rows took 2 ms; 0.27).
        uint32_t some_row = live;
        for (uint32_t left = __ballot_sync(~0u, row_max == 0u) & live; left; left &= left - 1) {
            const uint64_t r = first + __ffs(left) - 1;
            bool zero = true;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + j < a.cols) zero &= zero_factor<DT, SRC>(x + r * a.x_stride, grad_row(r), c0 + j, a.cols);
            if (__all_sync(~0u, zero)) some_row &= ~(left & -left);
        }
        if (T && lane == 0) some_rows[warp] = some_row;
#pragma unroll 1
        for (uint32_t left = __ballot_sync(~0u, at_border(row_max)) & some_row; left; left &= left - 1) {
            const int i = __ffs(left) - 1;
            const uint64_t r = first + i;
            double m = 0.0;
#pragma unroll 1
            for (int j = 0; j < 4; ++j)
                if (c0 + j < a.cols) m = fmax(m, source_magnitude<DT, SRC>(x + r * a.x_stride, grad_row(r), c0 + j, a.cols));
            __syncwarp();
#pragma unroll
            for (int d = 16; d; d >>= 1) m = fmax(m, __shfl_xor_sync(~0u, m, d));
            if (lane == i) row_max = settle(m);
        }
    }
    const uint32_t row_byte = scale_byte(row_max);
    const float row_inv = inverse_scale(row_byte);
    if (lane < kTileRows && first + lane < rows) a.scales[(uint64_t)col_tile * a.scales_stride + first + lane] = (uint8_t)row_byte;
    uint8_t* q = a.q + (uint64_t)first * a.q_stride + c0;
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        const float inv = __shfl_sync(~0u, row_inv, i);
        if (first + i < rows && c0 < a.cols) put_four(q + i * a.q_stride, to_e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3], inv), c0, a.cols);
    }
    if constexpr (T) {
        uint32_t m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m[j] = 0;
#pragma unroll
            for (int i = 0; i < kTileRows; ++i) m[j] = max(m[j], magnitude(v[i][j]));
        }
        *reinterpret_cast<uint4*>(&col_max[warp][lane * 4]) = make_uint4(m[0], m[1], m[2], m[3]);
        __syncthreads();
        if (threadIdx.x < 128) {  // a thread for each column
            const uint32_t c = col0 + threadIdx.x;
            uint32_t amax = 0;
#pragma unroll
            for (int w = 0; w < kTileThreads / 32; ++w) amax = max(amax, col_max[w][threadIdx.x]);
            if constexpr (SRC != CIERA_SOURCE_ROWS) {
                bool zero = c >= a.cols || amax == 0u;
                for (int w = 0; w < kTileThreads / 32 && __any_sync(~0u, zero && c < a.cols); ++w)
                    for (uint32_t rest = some_rows[w]; rest; rest &= rest - 1) {
                        const uint64_t r = row0 + w * kTileRows + __ffs(rest) - 1;
                        if (zero && c < a.cols)
                            zero = zero_factor<DT, SRC>(x + r * a.x_stride, SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + r * a.grad_stride : nullptr, c, a.cols);
                    }
                // the whole warp goes over such a column, four rows a lane
                for (uint32_t left = __ballot_sync(~0u, !zero && at_border(amax)); left; left &= left - 1) {
                    const int which = __ffs(left) - 1;
                    const uint32_t col = __shfl_sync(~0u, c, which);
                    double most = 0.0;
#pragma unroll 1
                    for (uint32_t r = row0 + lane; r < min(row0 + 128u, rows); r += 32) {
                        if (a.slot_of_row) {
                            const int32_t slot = a.slot_of_row[r];
                            if (slot < 0 || (uint64_t)slot >= a.x_rows * a.top_k) continue;
                        } else if (r >= a.x_rows) continue;
                        most = fmax(most, source_magnitude<DT, SRC>(x + (uint64_t)r * a.x_stride,
                                                                    SRC == CIERA_SOURCE_SWIGLU_BACKWARD ? grad + (uint64_t)r * a.grad_stride : nullptr, col, a.cols));
                    }
                    __syncwarp();
#pragma unroll
                    for (int d = 16; d; d >>= 1) most = fmax(most, __shfl_xor_sync(~0u, most, d));
                    if (lane == which) amax = settle(most);
                }
            }
            const uint32_t byte = scale_byte(amax);
            if (c < a.cols) a.scales_t[(uint64_t)row_tile * a.scales_t_stride + c] = (uint8_t)byte;
            col_inv[threadIdx.x] = inverse_scale(byte);
        }
        __syncthreads();
        const float4 inv4 = *reinterpret_cast<const float4*>(&col_inv[lane * 4]);
        const float inv[4] = {inv4.x, inv4.y, inv4.z, inv4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            turn_in(turned, lane, j, warp, to_e4m3x4(v[0][j], v[1][j], v[2][j], v[3][j], inv[j]), to_e4m3x4(v[4][j], v[5][j], v[6][j], v[7][j], inv[j]));
        __syncthreads();
        turn_out(turned, a.qt, a.qt_stride, col0, a.cols, row0, rows);
    }
}

// The 16-bit precisions as they are: a word of two values is halved into magnitudes and compared as it stands (their order is
// that of the bits), and a tile takes 16 registers a thread.  Half a warp has 4 rows, a lane 8 neighbouring columns of each: one
// access of 16 bytes, one of 8, and half the steps for each row that 4 columns a lane take (dispatch of 4096 x 8 rows of 2048
// as fp32 in the kernel above 81 us and 26 instructions a value, 4 columns of 16 bits a lane 74 us and 24).
constexpr uint32_t kMagnitudes = 0x7fff7fffu;

// the bits of the fp32 value that these magnitude bits stand for
template <int DT>
__device__ __forceinline__ uint32_t widen(uint32_t half) {
    if constexpr (DT == CIERA_BF16) return half << 16;
    else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)half)));
}
template <int DT>
__device__ __forceinline__ float2 two_values(uint32_t w) {
    if constexpr (DT == CIERA_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <int DT>
__device__ __forceinline__ uint32_t round_four(uint2 w, float inv) {
    const float2 a = two_values<DT>(w.x), b = two_values<DT>(w.y);
    return to_e4m3x4(a.x, a.y, b.x, b.y, inv);
}

__device__ __forceinline__ uint32_t most_of(uint4 w) {
    return max_two(max_two(w.x & kMagnitudes, w.y & kMagnitudes), max_two(w.z & kMagnitudes, w.w & kMagnitudes));
}
__device__ __forceinline__ uint4 most_of(uint4 a, uint4 b) {
    return make_uint4(max_two(a.x, b.x), max_two(a.y, b.y), max_two(a.z, b.z), max_two(a.w, b.w));
}
__device__ __forceinline__ uint4 magnitudes(uint4 w) {
    return make_uint4(w.x & kMagnitudes, w.y & kMagnitudes, w.z & kMagnitudes, w.w & kMagnitudes);
}

// A block an SM stays and takes neighbouring tiles one behind the other, with the next tile's values on their way (two blocks an SM
// with half the registers 63 us, a block for each tile 69, this 59).
template <int DT, bool T>
__global__ void __launch_bounds__(kTileThreads, 1) quantize_words_kernel(const RowsArgs a, const value_t<DT>* __restrict__ x) {
    __shared__ uint4 col_max[T ? kTileThreads / 32 : 1][16];
    __shared__ __align__(16) float col_inv[128];
    __shared__ __align__(16) uint32_t turned[T ? 128 * 32 : 4];
    pdl_wait();
    const uint32_t rows = a.starts ? min((uint32_t)max(a.starts[a.n_experts], 0), a.rows) : a.rows;
    const uint32_t tiles = (rows + 127) / 128 * a.col_tiles, each = (tiles + gridDim.x - 1) / gridDim.x;
    const uint32_t begin = min(tiles, blockIdx.x * each), end = min(tiles, begin + each);
    if (begin == end) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = lane >> 4, l16 = lane & 15;
    uint32_t row_tile = begin / a.col_tiles, col_tile = begin - row_tile * a.col_tiles;
    uint32_t from = 0, live = 0;
    const auto find_rows = [&](uint32_t tile) {  // lane i: where row i of the warp comes from
        from = tile * 128u + warp * kTileRows + lane;
        bool some = lane < kTileRows && from < rows;
        if (a.slot_of_row) {
            const int32_t slot = some ? a.slot_of_row[from] : -1;
            some = slot >= 0 && (uint64_t)slot < a.x_rows * a.top_k;
            from = (uint32_t)max(slot, 0) / a.top_k;
        } else {
            some = some && from < a.x_rows;
        }
        live = __ballot_sync(~0u, some) >> (4 * half);
    };
    uint4 coming[4];
    const auto fetch = [&](uint32_t tile) {
        const uint32_t c = tile * 128u + l16 * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = __shfl_sync(~0u, from, 4 * half + i);
            coming[i] = make_uint4(0, 0, 0, 0);
            if (c < a.cols && live >> i & 1) coming[i] = *reinterpret_cast<const uint4*>(x + r * a.x_stride + c);  // (cols: a multiple of 8)
        }
    };
    find_rows(row_tile);
    fetch(col_tile);
    for (uint32_t tile = begin; tile < end; ++tile) {
        const uint32_t row0 = row_tile * 128u, col0 = col_tile * 128u, row_t = row_tile, col_t = col_tile;
        const uint32_t c0 = col0 + l16 * 8, first = row0 + warp * kTileRows;
        const bool inside = c0 < a.cols;
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = coming[i];
        if (++col_tile == a.col_tiles) {
            col_tile = 0;
            ++row_tile;
            if (tile + 1 < end) find_rows(row_tile);
        }
        if (tile + 1 < end) fetch(col_tile);
        // the rows' largest magnitudes, two rows to a word
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t two = most_of(w[i]);
            m[i] = max(two >> 16, two & 0xffffu);
        }
        uint32_t m01 = m[0] | m[1] << 16, m23 = m[2] | m[3] << 16;
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            m01 = max_two(m01, __shfl_xor_sync(~0u, m01, d));
            m23 = max_two(m23, __shfl_xor_sync(~0u, m23, d));
        }
        const uint32_t pair = l16 & 2 ? m23 : m01;  // lane i of a half: row i & 3
        const uint32_t row_byte = scale_byte(widen<DT>(l16 & 1 ? pair >> 16 : pair & 0xffffu));
        const float row_inv = inverse_scale(row_byte);
        const uint32_t mine = first + 4 * half;  // the half's first row
        if (l16 < 4 && mine + l16 < rows) a.scales[(uint64_t)col_t * a.scales_stride + mine + l16] = (uint8_t)row_byte;
        uint8_t* q = a.q + (uint64_t)mine * a.q_stride + c0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float inv = __shfl_sync(~0u, row_inv, i, 16);
            const uint2 eight = make_uint2(round_four<DT>(make_uint2(w[i].x, w[i].y), inv), round_four<DT>(make_uint2(w[i].z, w[i].w), inv));
            if (mine + i < rows && inside) *reinterpret_cast<uint2*>(q + i * a.q_stride) = eight;
        }
        if constexpr (T) {
            uint4 cm = most_of(most_of(magnitudes(w[0]), magnitudes(w[1])), most_of(magnitudes(w[2]), magnitudes(w[3])));
            cm = most_of(cm, make_uint4(__shfl_xor_sync(~0u, cm.x, 16), __shfl_xor_sync(~0u, cm.y, 16), __shfl_xor_sync(~0u, cm.z, 16),
                                        __shfl_xor_sync(~0u, cm.w, 16)));
            if (!half) col_max[warp][l16] = cm;
            __syncthreads();
            if (threadIdx.x < 64) {  // a thread for two columns
                const uint32_t c = col0 + 2 * threadIdx.x;
                uint32_t two = 0;
#pragma unroll
                for (int i = 0; i < kTileThreads / 32; ++i) two = max_two(two, reinterpret_cast<const uint32_t*>(col_max[i])[threadIdx.x]);
                const uint32_t lo = scale_byte(widen<DT>(two & 0xffffu)), hi = scale_byte(widen<DT>(two >> 16));
                if (c < a.cols) {
                    a.scales_t[(uint64_t)row_t * a.scales_t_stride + c] = (uint8_t)lo;
                    a.scales_t[(uint64_t)row_t * a.scales_t_stride + c + 1] = (uint8_t)hi;
                }
                *reinterpret_cast<float2*>(&col_inv[2 * threadIdx.x]) = make_float2(inverse_scale(lo), inverse_scale(hi));
            }
            __syncthreads();
            // scaled by column, and the bytes turned: the four rows of a column are a word, at a place of its line that is mixed by the lane
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 inv = *reinterpret_cast<const float4*>(&col_inv[l16 * 8 + 4 * h]);
                uint32_t four[4], t[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 ab = two_values<DT>(h ? w[i].z : w[i].x), cd = two_values<DT>(h ? w[i].w : w[i].y);
                    four[i] = to_e4m3x4(ab.x, ab.y, cd.x, cd.y, inv);
                }
                turn_bytes(four[0], four[1], four[2], four[3], t);
#pragma unroll
                for (int j = 0; j < 4; ++j) turned[(l16 * 8 + 4 * h + j) * 32 + ((warp * 2 + half) ^ (l16 << 1))] = t[j];
            }
            __syncthreads();
            for (int k = threadIdx.x; k < 128 * 8; k += kTileThreads) {
                const uint32_t c = k >> 3, unit = k & 7, r = row0 + unit * 16, of = c >> 3;  // (the lane that put it there)
                if (col0 + c >= a.cols || r >= rows) continue;
                uint4 v = *reinterpret_cast<const uint4*>(turned + c * 32 + ((unit ^ (of >> 1)) << 2));
                if (of & 1) v = make_uint4(v.z, v.w, v.x, v.y);
                put_sixteen(a.qt + (uint64_t)(col0 + c) * a.qt_stride + r, v, r, rows);
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

template <int DT, bool T, bool WIDE>
__global__ void __launch_bounds__(kTileThreads, 2) quantize_blocks_kernel(const BlocksArgs a, const value_t<DT>* __restrict__ x) {
    __shared__ uint32_t warp_max[kTileThreads / 32];
    __shared__ __align__(16) uint2 turned[T ? 128 * 16 : 2];
    pdl_wait();
    const uint32_t row = blockIdx.x / a.col_blocks, cb = blockIdx.x - row * a.col_blocks;
    const uint32_t matrix = row / a.row_blocks, rb = row - matrix * a.row_blocks;
    const uint32_t row0 = rb * 128u, col0 = cb * 128u;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c0 = col0 + lane * 4, first = row0 + warp * kTileRows;
    const value_t<DT>* xm = x + matrix * a.x_matrix_stride;
    float v[kTileRows][4];
    uint32_t amax = 0, none = 0;
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = 0.f;
        if (first + i < a.rows && c0 < a.cols) {
            if constexpr (WIDE) load_values<DT, 4>(xm + (first + i) * a.x_stride + c0, v[i]);
            else source_values<DT, CIERA_SOURCE_ROWS>(xm + (first + i) * a.x_stride, nullptr, c0, a.cols, v[i], none);
        }
    }
#pragma unroll
    for (int i = 0; i < kTileRows; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) amax = max(amax, magnitude(v[i][j]));
    amax = __reduce_max_sync(~0u, amax);
    if (lane == 0) warp_max[warp] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTileThreads / 32; ++w) amax = max(amax, warp_max[w]);
    const uint32_t byte = scale_byte(amax);
    const float inv = inverse_scale(byte);
    if (threadIdx.x == 0) {
        a.scales[matrix * a.scales_matrix_stride + rb * a.scales_stride + cb] = (uint8_t)byte;
        if (T) a.scales_t[matrix * a.scales_t_matrix_stride + cb * a.scales_t_stride + rb] = (uint8_t)byte;
    }
    uint8_t* q = a.q + matrix * a.q_matrix_stride + c0;
    uint32_t four[kTileRows];
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        four[i] = to_e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3], inv);
        if (first + i < a.rows && c0 < a.cols) put_four(q + (first + i) * a.q_stride, four[i], c0, a.cols);
    }
    if constexpr (T) {  // (the same bytes)
        uint32_t lo[4], hi[4];
        turn_bytes(four[0], four[1], four[2], four[3], lo);
        turn_bytes(four[4], four[5], four[6], four[7], hi);
#pragma unroll
        for (int j = 0; j < 4; ++j) turn_in(turned, lane, j, warp, lo[j], hi[j]);
        __syncthreads();
        turn_out(turned, a.qt + matrix * a.qt_matrix_stride, a.qt_stride, col0, a.cols, row0, a.rows);
    }
}

template <int DT, bool T>
__global__ void __launch_bounds__(kTileThreads, 3) quantize_word_blocks_kernel(const BlocksArgs a, const value_t<DT>* __restrict__ x) {
    __shared__ uint32_t warp_max[kTileThreads / 32];
    __shared__ __align__(16) uint2 turned[T ? 128 * 16 : 2];
    pdl_wait();
    const uint32_t row = blockIdx.x / a.col_blocks, cb = blockIdx.x - row * a.col_blocks;
    const uint32_t matrix = row / a.row_blocks, rb = row - matrix * a.row_blocks;
    const uint32_t row0 = rb * 128u, col0 = cb * 128u;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c0 = col0 + lane * 4, first = row0 + warp * kTileRows;
    const value_t<DT>* xr = x + matrix * a.x_matrix_stride + first * a.x_stride + c0;
    const bool inside = c0 < a.cols;  // (cols is a multiple of four)
    uint2 w[kTileRows];
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        w[i] = make_uint2(0, 0);
        if (inside && first + i < a.rows) w[i] = *reinterpret_cast<const uint2*>(xr + i * a.x_stride);
    }
    uint32_t two = 0;
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) two = max_two(two, max_two(w[i].x & kMagnitudes, w[i].y & kMagnitudes));
    uint32_t amax = __reduce_max_sync(~0u, max(two >> 16, two & 0xffffu));
    if (lane == 0) warp_max[warp] = amax;
    __syncthreads();
    amax = __reduce_max_sync(~0u, warp_max[lane & 15]);
    const uint32_t byte = scale_byte(widen<DT>(amax));
    const float inv = inverse_scale(byte);
    if (threadIdx.x == 0) {
        a.scales[matrix * a.scales_matrix_stride + rb * a.scales_stride + cb] = (uint8_t)byte;
        if (T) a.scales_t[matrix * a.scales_t_matrix_stride + cb * a.scales_t_stride + rb] = (uint8_t)byte;
    }
    uint8_t* q = a.q + matrix * a.q_matrix_stride + first * a.q_stride + c0;
    uint32_t four[kTileRows];
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        four[i] = round_four<DT>(w[i], inv);
        if (inside && first + i < a.rows) *reinterpret_cast<uint32_t*>(q + i * a.q_stride) = four[i];
    }
    if constexpr (T) {
        uint32_t lo[4], hi[4];
        turn_bytes(four[0], four[1], four[2], four[3], lo);
        turn_bytes(four[4], four[5], four[6], four[7], hi);
#pragma unroll
        for (int j = 0; j < 4; ++j) turn_in(turned, lane, j, warp, lo[j], hi[j]);
        __syncthreads();
        turn_out(turned, a.qt + matrix * a.qt_matrix_stride, a.qt_stride, col0, a.cols, row0, a.rows);
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
    const uint64_t col_tiles = (p->cols + 127) / 128, tiles = (p->rows + 127) / 128 * col_tiles;
    if (tiles > kMaxExtent) return CIERA_ERR_UNSUPPORTED;
    // four values at a time where every row's start and, for gate and up, each half's is a multiple of four
    const uint64_t four = 4 * dtype_bytes(p->dtype) - 1;
    const bool wide = !(((uint64_t)p->x | (uint64_t)p->grad | p->x_stride * dtype_bytes(p->dtype) | p->grad_stride * dtype_bytes(p->dtype)) & four) &&
                      !(p->cols & (back ? 7 : 3));
    const RowsArgs a{p->x_stride, p->grad_stride, p->q_stride, p->scales_stride, p->qt_stride, p->scales_t_stride, p->x_rows,
                     p->slot_of_row, p->row_weights, p->starts, (uint32_t)p->rows, (uint32_t)p->cols, (uint32_t)col_tiles,
                     p->slot_of_row ? p->top_k : 1u, p->n_experts, (uint8_t*)p->q, p->scales, (uint8_t*)p->qt, p->scales_t};
    cudaError_t e = cudaSuccess;
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto go = [&](auto source, auto both, auto four_wide) {
            e = launch_after(quantize_rows_kernel<DT, decltype(source)::value, decltype(both)::value, decltype(four_wide)::value>, dim3((uint32_t)tiles),
                             kTileThreads, 0, (cudaStream_t)stream, a, (const value_t<DT>*)p->x, (const value_t<DT>*)p->grad);
        };
        if constexpr (DT != CIERA_FP32) {
            const bool eight = !(((uint64_t)p->x | p->x_stride * 2) & 15) && !(p->cols & 7);
            if (eight && src == CIERA_SOURCE_ROWS && !p->row_weights) {
                e = launch_after(turned ? quantize_words_kernel<DT, true> : quantize_words_kernel<DT, false>,
                                 dim3((uint32_t)(tiles < 148 ? tiles : 148)), kTileThreads, 0,
                                 (cudaStream_t)stream, a, (const value_t<DT>*)p->x);
                return;
            }
        }
        const auto pick = [&](auto source) {
            const std::true_type yes;
            const std::false_type no;
            if (turned) wide ? go(source, yes, yes) : go(source, yes, no);
            else wide ? go(source, no, yes) : go(source, no, no);
        };
        if (src == CIERA_SOURCE_ROWS) pick(std::integral_constant<int, CIERA_SOURCE_ROWS>());
        else if (!back) pick(std::integral_constant<int, CIERA_SOURCE_SWIGLU>());
        else pick(std::integral_constant<int, CIERA_SOURCE_SWIGLU_BACKWARD>());
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
    if (rb * p->matrices > kMaxExtent || rb * p->matrices * cb > kMaxExtent) return CIERA_ERR_UNSUPPORTED;
    const uint64_t v = dtype_bytes(p->dtype);
    const bool wide = !(((uint64_t)p->x | p->x_stride * v | p->x_matrix_stride * v) & (4 * v - 1)) && !(p->cols & 3);
    const BlocksArgs a{p->x_stride, p->x_matrix_stride, p->q_stride, p->q_matrix_stride, p->scales_stride, p->scales_matrix_stride,
                       p->qt_stride, p->qt_matrix_stride, p->scales_t_stride, p->scales_t_matrix_stride,
                       (uint32_t)p->rows, (uint32_t)p->cols, (uint32_t)rb, (uint32_t)cb, (uint8_t*)p->q, p->scales, (uint8_t*)p->qt, p->scales_t};
    cudaError_t e = cudaSuccess;
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto go = [&](auto both, auto four_wide) {
            e = launch_after(quantize_blocks_kernel<DT, decltype(both)::value, decltype(four_wide)::value>, dim3((uint32_t)(rb * p->matrices * cb)),
                             kTileThreads, 0, (cudaStream_t)stream, a, (const value_t<DT>*)p->x);
        };
        const std::true_type yes;
        const std::false_type no;
        if constexpr (DT != CIERA_FP32) {
            if (wide) {
                e = launch_after(turned ? quantize_word_blocks_kernel<DT, true> : quantize_word_blocks_kernel<DT, false>,
                                 dim3((uint32_t)(rb * p->matrices * cb)), kTileThreads, 0, (cudaStream_t)stream, a, (const value_t<DT>*)p->x);
            } else {
                turned ? go(yes, no) : go(no, no);
            }
        } else {
            if (turned) wide ? go(yes, yes) : go(yes, no);
            else wide ? go(no, yes) : go(no, no);
        }
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
