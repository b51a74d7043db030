// Operands of the 4-bit products: rows or matrices rounded to e2m1 with a power of two for each 32 values of a row, and back.
//
// A lane has 8 neighbouring columns, so a group of 32 belongs to four neighbouring lanes and a row of 256 columns to a warp; its
// largest magnitude is two exchanges, its codes are one word a lane.  A warp takes rows r, r + 32, r + 64 and r + 96 of an atom of
// scales together: their scale bytes are 16 neighbouring bytes of the atom, and their loads are on their way at the same time.
// Transposed matrices go through shared memory, two columns to a word.
#include <type_traits>

#include "ciera_fp4.cuh"
#include "ciera_swiglu.cuh"

namespace ciera {

constexpr int kFp4Threads = 256;

// 2^-s; 0 for byte 255
__device__ __forceinline__ float inverse_scale4(uint32_t byte) { return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23); }
__device__ __forceinline__ uint32_t magnitude4(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Two values as a byte, the first in the low half.
__device__ __forceinline__ uint32_t to_e2m1x2(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 a;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.u32.u8 %0, a;\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}
// Eight values, the first in the lowest four bits.
__device__ __forceinline__ uint32_t to_e2m1x8(const float (&v)[8], float inv) {
    const uint32_t a = to_e2m1x2(v[0] * inv, v[1] * inv), b = to_e2m1x2(v[2] * inv, v[3] * inv);
    const uint32_t c = to_e2m1x2(v[4] * inv, v[5] * inv), d = to_e2m1x2(v[6] * inv, v[7] * inv);
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// ---- 256 values of a row, eight neighbouring ones a lane, as they are in memory

// Rows that start at multiples of 16 bytes and are multiples of 8 wide: the lane's own.  Others: words of 4 bytes, neighbouring ones
// by neighbouring lanes, that go through the warp's shared memory.  (Eight accesses of 2 bytes a lane: silu(g) * u of 8008 rows of
// 1001 35 us, their values back 50 us; so 31 and 18.)
template <int DT>
constexpr int kWords = 8 * sizeof(value_t<DT>) / 4;  // of a lane
template <int DT>
struct Staging {
    uint32_t w[kWords<DT> * 32 + 4];
};

template <int DT, bool WIDE>
struct RawEight {
    uint32_t w[kWords<DT>];
    uint32_t last;  // (not WIDE, 16 bits: lane 0's, the one behind the lanes')

    // n: values of the row from the warp's first on, more than 0
    __device__ __forceinline__ void load(const value_t<DT>* __restrict__ at, uint32_t n, int lane) {
        if constexpr (WIDE) {
            if (lane * 8u >= n) {
#pragma unroll
                for (int i = 0; i < kWords<DT>; ++i) w[i] = 0;
            } else {
                const uint4* from = reinterpret_cast<const uint4*>(at + lane * 8);
#pragma unroll
                for (int i = 0; i < kWords<DT>; i += 4) {
                    const uint4 v = __ldg(from + i / 4);
                    w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
                }
            }
        } else if constexpr (DT == CIERA_FP32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = lane + 32u * i < n ? __ldg(reinterpret_cast<const uint32_t*>(at) + lane + 32 * i) : 0u;
        } else {
            // values v0 = 2 * word - odd and v0 + 1, of which the first may be before and the second behind the row
            const int odd = (int)((uintptr_t)at >> 1 & 1u);
            const int count = (int)min(n, 256u);
            const auto word = [&](int i) -> uint32_t {
                const int v0 = 2 * i - odd;
                if (v0 >= 0 && v0 + 1 < count) return __ldg(reinterpret_cast<const uint32_t*>(at + v0));
                const unsigned short* h = reinterpret_cast<const unsigned short*>(at);
                uint32_t r = 0;
                if (v0 >= 0 && v0 < count) r = __ldg(h + v0);
                if (v0 + 1 >= 0 && v0 + 1 < count) r |= (uint32_t)__ldg(h + v0 + 1) << 16;
                return r;
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = word(lane + 32 * i);
            last = odd && lane == 0 ? word(128) : 0u;
        }
    }
    // by the whole warp
    __device__ __forceinline__ void get(const value_t<DT>* __restrict__ at, Staging<DT>& st, float (&v)[8], int lane) {
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < kWords<DT>; ++i) st.w[lane + 32 * i] = w[i];
            if (DT != CIERA_FP32 && lane == 0) st.w[32 * kWords<DT>] = last;
            __syncwarp();
            const uint4* from = reinterpret_cast<const uint4*>(st.w) + lane * (kWords<DT> / 4);
#pragma unroll
            for (int i = 0; i < kWords<DT>; i += 4) {
                const uint4 x = from[i / 4];
                w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
            }
            if (DT != CIERA_FP32 && ((uintptr_t)at >> 1 & 1u)) {
                const uint32_t next = st.w[lane * 4 + 4];
                w[0] = __byte_perm(w[0], w[1], 0x5432);
                w[1] = __byte_perm(w[1], w[2], 0x5432);
                w[2] = __byte_perm(w[2], w[3], 0x5432);
                w[3] = __byte_perm(w[3], next, 0x5432);
            }
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DT == CIERA_FP32) v[i] = __uint_as_float(w[i]);
            else if constexpr (DT == CIERA_BF16) v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
            else v[i] = __half2float(__ushort_as_half((unsigned short)(w[i / 2] >> (16 * (i & 1)))));
        }
    }
};

struct Rows4Args {
    uint64_t x_stride, x_matrix_stride, q_stride, q_matrix_stride, scales_stride, scales_matrix_stride;
    uint64_t x_rows;
    const int32_t* slot_of_row;
    const int32_t* starts;
    uint32_t rows, cols, col_tiles, units, each, chunks, top_k, n_experts, source_rows;  // units: warps of a matrix; tiles of each; chunks of a line
    uint8_t* q;
    uint8_t* scales;
};

// A largest magnitude of silu(g) * u that 32 bits do not settle: within 256 steps of the border 1.5 * 2^n (they are off by less than
// 2^-20), or so small that a factor has left their range.
__device__ __forceinline__ bool at_border4(uint32_t amax) {
    return amax < 0x7f800000u && (amax < (32u << 23) || (uint32_t)((amax & 0x7fffffu) - 0x400000u + 256u) <= 512u);
}

// A warp takes rows r + 32 * j of a block of 128 and `each` neighbouring tiles of 256 columns; the next rows' values are on their way
// (four, or two of gates and ups, which take twice the registers).
template <int DT, int SRC, bool WIDE>
__global__ void __launch_bounds__(kFp4Threads, SRC == CIERA_SOURCE_SWIGLU ? 3 : 4) quantize4_rows_kernel(const Rows4Args a, const value_t<DT>* __restrict__ x_) {
    constexpr bool kSwiglu = SRC == CIERA_SOURCE_SWIGLU;
    constexpr int kAhead = kSwiglu || DT == CIERA_FP32 ? 2 : 4;
    __shared__ __align__(16) Staging<DT> staging[WIDE ? 1 : kFp4Threads / 32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t used = a.starts ? min((uint32_t)max(a.starts[a.n_experts], 0), a.rows) : a.rows;
    const uint32_t unit = blockIdx.x * (kFp4Threads / 32) + warp;
    if (unit >= a.units) return;
    const uint32_t line = unit / a.chunks, tile0 = (unit - line * a.chunks) * a.each, tile1 = min(tile0 + a.each, a.col_tiles);
    const uint32_t rb = line >> 5, r0 = rb * 128u + (line & 31u);
    if (r0 >= used) return;
    Staging<DT>& st = staging[WIDE ? 0 : warp];
    const value_t<DT>* at[4];  // the rows' first tile
    uint32_t there;            // bit j: row j comes from anywhere
    {
        const uint32_t row = r0 + 32u * (lane & 3);
        bool some = row < used;
        uint32_t from = row;
        if (a.slot_of_row) {
            const int32_t slot = some ? __ldg(a.slot_of_row + row) : -1;
            some = slot >= 0 && (uint64_t)slot < a.x_rows * a.top_k;
            if (!kSwiglu) from = some ? (uint32_t)slot / a.top_k : 0u;
        }
        there = __ballot_sync(~0u, some) & 15u;
#pragma unroll
        for (int j = 0; j < 4; ++j) at[j] = x_ + blockIdx.y * a.x_matrix_stride + (uint64_t)__shfl_sync(~0u, from, j) * a.x_stride + tile0 * 256u;
    }
    uint8_t* q = a.q + blockIdx.y * a.q_matrix_stride + (uint64_t)r0 * a.q_stride + tile0 * 128u + lane * 4;
    RawEight<DT, WIDE> raw[kAhead], raw_up[kSwiglu ? kAhead : 1];
    const auto load = [&](int to, int j, uint32_t tile) {  // row j's tile
        if (tile < tile1 && (there >> j & 1u)) {
            const value_t<DT>* p = at[j] + (tile - tile0) * 256u;
            raw[to].load(p, a.cols - tile * 256u, lane);
            if constexpr (kSwiglu) raw_up[to].load(p + a.cols, a.cols - tile * 256u, lane);
        }
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) load(j, j, tile0);
    for (uint32_t tile = tile0; tile < tile1; ++tile, q += 128) {
        const uint32_t c0 = tile * 256u + lane * 8;
        uint32_t bytes = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            constexpr int A = kAhead;
            const uint32_t row = r0 + 32u * j;
            uint32_t codes = 0, byte = 127u;
            if (there >> j & 1u) {
                const value_t<DT>* p = at[j] + (tile - tile0) * 256u;
                float v[8];
                uint32_t amax = 0;
                raw[j % A].get(p, st, v, lane);
                bool some = false;  // a value is more than a zero times something
                if constexpr (kSwiglu) {
                    float u[8];
                    raw_up[j % A].get(p + a.cols, st, u, lane);
                    bool low = false;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float g = v[i];
                        low |= g < kLowestGate;
                        some |= g != 0.f && u[i] != 0.f;
                        v[i] = swiglu32_any(g, u[i]);
                    }
                    if (low) {
#pragma unroll 1
                        for (int i = 0; i < 8; ++i)
                            if (c0 + i < a.cols) {
                                const double g = ValueOf<DT>::get(p[lane * 8 + i]);
                                const float y = (float)(g / (1.0 + exp(-g)) * (double)ValueOf<DT>::get(p[a.cols + lane * 8 + i]));
#pragma unroll
                                for (int k = 0; k < 8; ++k)
                                    if (k == i && g < (double)kLowestGate) v[k] = y;
                            }
                    }
                }
                load(j % A, (j + A) & 3, tile + ((j + A) >> 2));
#pragma unroll
                for (int i = 0; i < 8; ++i) amax = max(amax, magnitude4(v[i]));
                amax = max(amax, __shfl_xor_sync(~0u, amax, 1));
                amax = max(amax, __shfl_xor_sync(~0u, amax, 2));
                if constexpr (kSwiglu) {
                    // settled in 64 bits, by the four lanes of each such group
                    const uint32_t has = __ballot_sync(~0u, some) >> (lane & 28) & 15u;
                    const bool settle = at_border4(amax) && has;
                    if (__any_sync(~0u, settle)) {
                        double most = 0.0;
                        if (settle) {
#pragma unroll 1
                            for (uint32_t c = 0; c < 8 && c0 + c < a.cols; ++c) {
                                const double g = ValueOf<DT>::get(p[lane * 8 + c]), u = ValueOf<DT>::get(p[a.cols + lane * 8 + c]);
                                most = fmax(most, fabs(g / (1.0 + exp(-g)) * u));
                            }
                        }
                        most = fmax(most, __shfl_xor_sync(~0u, most, 1));
                        most = fmax(most, __shfl_xor_sync(~0u, most, 2));
                        if (settle) amax = __float_as_uint(__double2float_ru(most));
                    }
                }
                byte = scale_byte4(amax);
                codes = to_e2m1x8(v, inverse_scale4(byte));
                if (byte == 255u) codes = 0u;
            } else {
                load(j % A, (j + A) & 3, tile + ((j + A) >> 2));
            }
            bytes |= byte << (8 * j);
            if (row < used && c0 < a.cols) {
                uint8_t* to = q + 32 * j * a.q_stride;
                if (c0 + 8 <= a.cols) {
                    *reinterpret_cast<uint32_t*>(to) = codes;
                } else {
                    for (uint32_t i = 0; 2 * i < a.cols - c0; ++i) to[i] = (uint8_t)(codes >> (8 * i));
                }
            }
        }
        // from a group's bytes of four rows to a row's of four groups, which lane 4 * j of the 16 writes for row j
        const uint32_t g = lane >> 2;
        uint32_t t = __shfl_xor_sync(~0u, bytes, 4);
        bytes = g & 1 ? __byte_perm(t, bytes, 0x7351) : __byte_perm(bytes, t, 0x6240);
        t = __shfl_xor_sync(~0u, bytes, 8);
        bytes = g & 2 ? __byte_perm(t, bytes, 0x7632) : __byte_perm(bytes, t, 0x5410);
        const uint32_t row = r0 + 32u * (g & 3), atom = tile * 2 + (lane >> 4);
        if (!(lane & 3) && row < used && atom * 128u < a.cols)
            *reinterpret_cast<uint32_t*>(a.scales + blockIdx.y * a.scales_matrix_stride + (uint64_t)rb * a.scales_stride + (uint64_t)atom * kAtomBytes +
                                         atom_word(row)) = bytes;
    }
}

// The same for rows of 16-bit values that lie in whole pieces of 16 bytes, which are compared as they are, two at a time.  What four
// lanes need for each of four rows, the largest magnitude and the scale, each of them works out for one: 330 instructions for 4 rows
// of 256 instead of 460, and 32768 rows of 2048 in 34 us instead of 42.
template <int DT>
__global__ void __launch_bounds__(kFp4Threads, 4) quantize4_words_kernel(const Rows4Args a, const value_t<DT>* __restrict__ x) {
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t used = a.starts ? min((uint32_t)max(a.starts[a.n_experts], 0), a.rows) : a.rows;
    const uint32_t unit = blockIdx.x * (kFp4Threads / 32) + warp;
    if (unit >= a.units) return;
    const uint32_t line = unit / a.chunks, tile0 = (unit - line * a.chunks) * a.each, tile1 = min(tile0 + a.each, a.col_tiles);
    const uint32_t rb = line >> 5, r0 = rb * 128u + (line & 31u);
    if (r0 >= used) return;
    const uint32_t mine = r0 + 32u * (lane & 3);  // the lane's of the four rows
    uint32_t from = mine;
    bool some = mine < used;
    if (a.slot_of_row) {
        const int32_t slot = some ? __ldg(a.slot_of_row + mine) : -1;
        some = slot >= 0 && (uint64_t)slot < a.x_rows * a.top_k;
        from = some ? (uint32_t)slot / a.top_k : 0u;
    }
    const uint32_t there = __ballot_sync(~0u, some) & 15u, rows_there = __ballot_sync(~0u, mine < used) & 15u;
    const uint4* at[4];
    uint8_t* q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        at[j] = reinterpret_cast<const uint4*>(x + blockIdx.y * a.x_matrix_stride + (uint64_t)__shfl_sync(~0u, from, j) * a.x_stride) + tile0 * 32u + lane;
        q[j] = a.q + blockIdx.y * a.q_matrix_stride + (uint64_t)(r0 + 32u * j) * a.q_stride + tile0 * 128u + lane * 4;
    }
    uint8_t* scales = a.scales + blockIdx.y * a.scales_matrix_stride + (uint64_t)rb * a.scales_stride + (uint64_t)(tile0 * 2 + (lane >> 4)) * kAtomBytes + atom_word(mine);
    const auto fetch = [&](uint4 (&w)[4], uint32_t tile) {
        const bool inside = tile * 256u + lane * 8 < a.cols;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = make_uint4(0, 0, 0, 0);
            if (inside && (there >> j & 1u)) w[j] = __ldg(at[j] + (tile - tile0) * 32u);
        }
    };
    // the larger of two magnitudes, of two halves at a time; a NaN stays one; signs do not matter
    const auto two = [](uint32_t l, uint32_t r) {
        uint32_t m;
        if constexpr (DT == CIERA_BF16) asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(l), "r"(r));
        else asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(m) : "r"(l), "r"(r));
        return m;
    };
    uint4 w[4], next[4];
    fetch(w, tile0);
    for (uint32_t tile = tile0; tile < tile1; ++tile) {
        if (tile + 1 < tile1) fetch(next, tile + 1);
        uint32_t m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = two(two(w[j].x, w[j].y), two(w[j].z, w[j].w));
        const uint32_t odd = lane & 1, high = lane & 2;
        const uint32_t m0 = two(odd ? m[1] : m[0], __shfl_xor_sync(~0u, odd ? m[0] : m[1], 1));
        const uint32_t m1 = two(odd ? m[3] : m[2], __shfl_xor_sync(~0u, odd ? m[2] : m[3], 1));
        uint32_t amax = two(high ? m1 : m0, __shfl_xor_sync(~0u, high ? m0 : m1, 2));
        amax = two(amax, amax << 16) & 0x7fff0000u;
        if constexpr (DT == CIERA_FP16) amax = __float_as_uint(__half2float(__ushort_as_half((unsigned short)(amax >> 16))));
        const uint32_t byte = scale_byte4(amax), inverse = __float_as_uint(inverse_scale4(byte));
        uint32_t word = byte << (lane * 2 & 24);
        word |= __shfl_xor_sync(~0u, word, 4);
        word |= __shfl_xor_sync(~0u, word, 8);
        if (!(lane & 12) && mine < used && tile * 256u + (lane & 16) * 8 < a.cols) *reinterpret_cast<uint32_t*>(scales + (uint64_t)(tile - tile0) * (2 * kAtomBytes)) = word;
        const bool inside = tile * 256u + lane * 8 < a.cols;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t inv = __shfl_sync(~0u, inverse, (lane & 28) + j);
            const uint32_t x4[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
            uint32_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (DT == CIERA_BF16) {  // (by a power of two: exact, but for what is far below the least code)
                    const uint32_t both = __byte_perm(inv, 0, 0x3232);
                    const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x4[i]), *reinterpret_cast<const __nv_bfloat162*>(&both));
                    const uint32_t bits = *reinterpret_cast<const uint32_t*>(&y);
                    c[i] = to_e2m1x2(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u));
                } else {
                    const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&x4[i]));
                    c[i] = to_e2m1x2(y.x * __uint_as_float(inv), y.y * __uint_as_float(inv));
                }
            }
            uint32_t codes = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
            if (inv == 0u) codes = 0u;
            if (inside && (rows_there >> j & 1u)) *reinterpret_cast<uint32_t*>(q[j] + (tile - tile0) * 128u) = codes;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = next[j];
    }
}

struct Turned4Args {
    uint64_t x_stride, x_matrix_stride, q_stride, q_matrix_stride, scales_stride, scales_matrix_stride;
    uint32_t rows, cols, row_tiles, col_tiles;
    uint8_t* q;
    uint8_t* scales;
};

// Transposed: a block has 128 rows (the contraction) and 256 bytes of columns, 64 words of two 16-bit columns or one of 32 bits.
// A thread rounds the 32 values of a group in its word's columns; word w of row r lies at (w + 8 * (r / 32)) % 64, so that the four
// groups of 8 words, which a warp reads together, are in different banks.
template <int DT, bool WIDE>
__global__ void __launch_bounds__(kFp4Threads) quantize4_turned_kernel(const Turned4Args a, const value_t<DT>* __restrict__ x_) {
    constexpr int kCols = 4 / sizeof(value_t<DT>);  // of a word
    __shared__ __align__(16) uint32_t tile[128 * 64];
    pdl_wait();
    const uint32_t row_tile = blockIdx.x % a.row_tiles, col_tile = blockIdx.x / a.row_tiles;
    const uint32_t row0 = row_tile * 128u, col0 = col_tile * 64u * kCols;
    const value_t<DT>* x = x_ + blockIdx.y * a.x_matrix_stride;
    if (WIDE) {
        uint4 v[8];
        const uint32_t piece = threadIdx.x & 15, c = col0 + piece * 4 * kCols;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = row0 + i * 16 + (threadIdx.x >> 4);
            v[i] = make_uint4(0, 0, 0, 0);
            if (r < a.rows && c < a.cols) v[i] = *reinterpret_cast<const uint4*>(x + (uint64_t)r * a.x_stride + c);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = i * 16 + (threadIdx.x >> 4);
            *reinterpret_cast<uint4*>(tile + r * 64 + ((piece * 4 + 8 * (r >> 5)) & 63)) = v[i];
        }
    } else {
        // words of 4 bytes, neighbouring ones by neighbouring lanes, 16 rows a warp; a row that starts in the middle of one is shifted on the
        // way.  (Value by value: 27 matrices of 1373 x 1374 in 126 us with the values back, 102 so.)
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int count = (int)min(a.cols - col0, 64u * kCols);
#pragma unroll 1
        for (int i0 = 0; i0 < 16; i0 += 4) {
            uint32_t v[4][3];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t r = warp * 16 + i0 + i;
                const bool here = row0 + r < a.rows;
                const value_t<DT>* at = x + (uint64_t)(row0 + r) * a.x_stride + col0;
                const int odd = DT == CIERA_FP32 ? 0 : (int)((uintptr_t)at >> 1 & 1u);
                const auto word = [&](int k) -> uint32_t {
                    const int v0 = k * kCols - odd;
                    if (!here) return 0;
                    if constexpr (DT == CIERA_FP32) return v0 < count ? __ldg(reinterpret_cast<const uint32_t*>(at) + v0) : 0u;
                    if (v0 >= 0 && v0 + 1 < count) return __ldg(reinterpret_cast<const uint32_t*>(at + v0));
                    const unsigned short* h = reinterpret_cast<const unsigned short*>(at);
                    uint32_t b = 0;
                    if (v0 >= 0 && v0 < count) b = __ldg(h + v0);
                    if (v0 + 1 >= 0 && v0 + 1 < count) b |= (uint32_t)__ldg(h + v0 + 1) << 16;
                    return b;
                };
                v[i][0] = word(lane);
                v[i][1] = word(lane + 32);
                v[i][2] = odd && lane == 0 ? word(64) : 0u;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t r = warp * 16 + i0 + i, turn = 8 * (r >> 5);
                uint32_t lo = v[i][0], hi = v[i][1];
                if constexpr (DT != CIERA_FP32) {
                    const value_t<DT>* at = x + (uint64_t)(row0 + r) * a.x_stride + col0;
                    if ((uintptr_t)at >> 1 & 1u) {
                        const uint32_t first = __shfl_sync(~0u, hi, 0), last = __shfl_sync(~0u, v[i][2], 0);
                        const uint32_t lo1 = __shfl_down_sync(~0u, lo, 1), hi1 = __shfl_down_sync(~0u, hi, 1);
                        lo = __byte_perm(lo, lane == 31 ? first : lo1, 0x5432);
                        hi = __byte_perm(hi, lane == 31 ? last : hi1, 0x5432);
                    }
                }
                tile[r * 64 + ((lane + turn) & 63)] = lo;
                tile[r * 64 + ((lane + 32 + turn) & 63)] = hi;
            }
        }
    }
    __syncthreads();
    const uint32_t group = threadIdx.x & 3, w = threadIdx.x >> 2;
    const uint32_t* from = tile + group * 32 * 64 + ((w + 8 * group) & 63);
    uint32_t word[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) word[i] = from[i * 64];
    uint32_t bytes[kCols];
#pragma unroll
    for (int k = 0; k < kCols; ++k) {
        const auto value = [&](int i) {
            if constexpr (DT == CIERA_FP32) return __uint_as_float(word[i]);
            else if constexpr (DT == CIERA_BF16) return __uint_as_float(k ? word[i] & 0xffff0000u : word[i] << 16);
            else return __half2float(__ushort_as_half((unsigned short)(word[i] >> (16 * k))));
        };
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) amax = max(amax, magnitude4(value(i)));
        const uint32_t byte = bytes[k] = scale_byte4(amax);
        const float inv = inverse_scale4(byte);
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v[8] = {value(8 * i), value(8 * i + 1), value(8 * i + 2), value(8 * i + 3),
                                value(8 * i + 4), value(8 * i + 5), value(8 * i + 6), value(8 * i + 7)};
            q[i] = byte == 255u ? 0u : to_e2m1x8(v, inv);
        }
        const uint32_t c = col0 + w * kCols + k, r = row0 + group * 32;
        if (c < a.cols && r < a.rows) {
            uint8_t* to = a.q + blockIdx.y * a.q_matrix_stride + (uint64_t)c * a.q_stride + r / 2;
            if (r + 32 <= a.rows) {
                *reinterpret_cast<uint4*>(to) = make_uint4(q[0], q[1], q[2], q[3]);
            } else {
                for (uint32_t i = 0; 2 * i < a.rows - r; ++i) {
                    const uint32_t part = i < 4 ? q[0] : i < 8 ? q[1] : i < 12 ? q[2] : q[3];
                    to[i] = (uint8_t)(part >> (8 * (i & 3)));
                }
            }
        }
    }
    // four neighbouring lanes have a column's four groups
#pragma unroll
    for (int k = 0; k < kCols; ++k) {
        uint32_t all = bytes[k] << (8 * group);
        all |= __shfl_xor_sync(~0u, all, 1);
        all |= __shfl_xor_sync(~0u, all, 2);
        const uint32_t c = col0 + w * kCols + k;
        if (group == 0 && c < a.cols)
            *reinterpret_cast<uint32_t*>(a.scales + blockIdx.y * a.scales_matrix_stride + (uint64_t)(c >> 7) * a.scales_stride + (uint64_t)row_tile * kAtomBytes +
                                         atom_word(c)) = all;
    }
}

struct Values4Args {
    uint64_t q_stride, q_matrix_stride, scales_stride, scales_matrix_stride, out_stride, out_matrix_stride;
    uint32_t rows, cols, col_tiles, units;
    const uint8_t* q;
    const uint8_t* scales;
};

// Back: the same rows and columns for a warp as above.
template <int DT, bool WIDE>
__global__ void __launch_bounds__(kFp4Threads) values4_kernel(const Values4Args a, value_t<DT>* __restrict__ out_) {
    __shared__ __align__(16) Staging<DT> staging[WIDE ? 1 : kFp4Threads / 32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t unit = blockIdx.x * (kFp4Threads / 32) + warp;
    if (unit >= a.units) return;
    const uint32_t line = unit / a.col_tiles, tile = unit - line * a.col_tiles;
    const uint32_t rb = line >> 5, r0 = rb * 128u + (line & 31u), c0 = tile * 256u + lane * 8;
    const bool inside = c0 < a.cols;
    if (r0 >= a.rows || (WIDE && !inside)) return;
    Staging<DT>& st = staging[WIDE ? 0 : warp];
    const uint8_t* q = a.q + blockIdx.y * a.q_matrix_stride + c0 / 2;
    uint4 s = make_uint4(0, 0, 0, 0);
    if (inside) s = *reinterpret_cast<const uint4*>(a.scales + blockIdx.y * a.scales_matrix_stride + (uint64_t)rb * a.scales_stride +
                                                    (uint64_t)(c0 >> 7) * kAtomBytes + (line & 31u) * 16);
    const uint32_t scale[4] = {s.x, s.y, s.z, s.w};
    uint32_t codes[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t row = r0 + 32u * j;
        codes[j] = 0;
        if (row >= a.rows || !inside) continue;
        const uint8_t* from = q + (uint64_t)row * a.q_stride;
        if (c0 + 8 <= a.cols) {
            codes[j] = *reinterpret_cast<const uint32_t*>(from);
        } else {
            for (uint32_t i = 0; 2 * i < a.cols - c0; ++i) codes[j] |= (uint32_t)from[i] << (8 * i);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t row = r0 + 32u * j;
        if (row >= a.rows) continue;
        const float f = scale_value(scale[j] >> (lane >> 2 & 3) * 8 & 255u);
        float v[8];
        uint32_t two[4];
        from_e2m1x8(codes[j], two);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&two[i]));
            v[2 * i] = y.x * f;
            v[2 * i + 1] = y.y * f;
        }
        value_t<DT>* line_at = out_ + blockIdx.y * a.out_matrix_stride + (uint64_t)row * a.out_stride + tile * 256u;
        if constexpr (WIDE) {
            value_t<DT>* to = line_at + lane * 8;
            if (c0 + 8 <= a.cols) {
                constexpr int kEach = 16 / sizeof(value_t<DT>);
#pragma unroll
                for (int i = 0; i < 8; i += kEach) {
                    float part[kEach];
#pragma unroll
                    for (int k = 0; k < kEach; ++k) part[k] = v[i + k];
                    store_values<DT, kEach>(to + i, part);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0 + i < a.cols) to[i] = ValueOf<DT>::put(v[i]);
            }
        } else {
            // through shared memory to neighbouring words by neighbouring lanes, as they are read
            const uint32_t n = min(a.cols - tile * 256u, 256u);
            Pack<value_t<DT>, 16 / sizeof(value_t<DT>)>* put = reinterpret_cast<Pack<value_t<DT>, 16 / sizeof(value_t<DT>)>*>(st.w) + lane * (kWords<DT> / 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) put[i * sizeof(value_t<DT>) / 16].v[i % (16 / sizeof(value_t<DT>))] = ValueOf<DT>::put(v[i]);
            __syncwarp();
            if constexpr (DT == CIERA_FP32) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (lane + 32u * i < n) reinterpret_cast<uint32_t*>(line_at)[lane + 32 * i] = st.w[lane + 32 * i];
            } else {
                const int odd = (int)((uintptr_t)line_at >> 1 & 1u), count = (int)n;
                const unsigned short* h = reinterpret_cast<const unsigned short*>(st.w);
                const auto write = [&](int i) {
                    const int v0 = 2 * i - odd;
                    if (v0 >= 0 && v0 + 1 < count) {
                        *reinterpret_cast<uint32_t*>(line_at + v0) = odd ? __byte_perm(st.w[i - 1], st.w[i], 0x5432) : st.w[i];
                        return;
                    }
                    unsigned short* to = reinterpret_cast<unsigned short*>(line_at);
                    if (v0 >= 0 && v0 < count) to[v0] = h[v0];
                    if (v0 + 1 >= 0 && v0 + 1 < count) to[v0 + 1] = h[v0 + 1];
                };
#pragma unroll
                for (int i = 0; i < 4; ++i) write(lane + 32 * i);
                if (odd && lane == 0) write(128);
            }
            __syncwarp();
        }
    }
}

// An operand's codes and scales; lines: of atoms.  0, or the status of what is wrong with them.
static int operand4(const void* q, uint64_t q_stride, uint64_t q_matrix_stride, const void* scales, uint64_t scales_stride,
                    uint64_t scales_matrix_stride, uint64_t matrices, uint64_t rows, uint64_t cols) {
    const uint64_t line = (cols + 1) / 2, atoms = (cols + 127) / 128;
    if (!q || !scales || (rows > 1 && q_stride < line) || (rows > 128 && scales_stride < atoms * kAtomBytes)) return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(q, 16) || !aligned_to(scales, 16) || (rows > 1 && (q_stride & 15)) || (rows > 128 && (scales_stride & 511)) ||
        (matrices > 1 && ((q_matrix_stride | scales_matrix_stride) & 15)))
        return CIERA_ERR_MISALIGNED;
    return CIERA_OK;
}

// (a tile of a line each)
static uint64_t warp_units(uint64_t rows, uint64_t cols) {
    return (rows + 127) / 128 * (rows < 32 ? rows : 32) * ((cols + 255) / 256);
}

// Warps' work: 32 lines for each block of 128 rows (of a single block with fewer rows those that it has), whole if that leaves `warps`
// warps for each of the 148 SMs over the whole call, else in pieces.  Long pieces have the next tile's values on their way, short ones end
// together: 24 for rows as they are, which have four rows ahead (32768 gathered rows of 2048 29.7 us, with 48 29.9, with 96 32.2), 96 for
// silu(g) * u, which has two and more to do for each (8008 rows of 1001 27.2 us, with 48 30.1; 32768 of 1024 50.7, with 48 52.1, with 192 54.8).
constexpr uint32_t kRowWarps = 24, kSwigluWarps = 96;
static uint64_t rows_units(uint64_t rows, uint64_t cols, uint64_t matrices, uint32_t* each, uint32_t* chunks, uint32_t warps) {
    const uint64_t tiles = (cols + 255) / 256, lines = (rows + 127) / 128 * (rows < 32 ? rows : 32);
    const uint64_t most = lines * tiles * matrices / (148 * warps);
    *each = (uint32_t)(most < 1 ? 1 : most > tiles ? tiles : most);
    *chunks = (uint32_t)((tiles + *each - 1) / *each);
    return lines * *chunks;
}

template <int SRC>
static cudaError_t launch_rows4(const Rows4Args& a, int dtype, const void* x, uint32_t matrices, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const uint64_t v = dtype_bytes(DT);
        uint64_t at = (uint64_t)x | (a.source_rows > 1 ? a.x_stride * v : 0) | (matrices > 1 ? a.x_matrix_stride * v : 0);
        if (SRC == CIERA_SOURCE_SWIGLU) at |= a.cols * v;
        const dim3 grid((a.units + kFp4Threads / 32 - 1) / (kFp4Threads / 32), matrices);
        // (rows of whole pieces of 16 bytes)
        const bool wide = !((at | (uint64_t)a.cols * v) & 15) && !(a.cols & 7);
        if constexpr (SRC == CIERA_SOURCE_ROWS && DT != CIERA_FP32) {
            if (wide) {
                e = launch_after(quantize4_words_kernel<DT>, grid, kFp4Threads, 0, s, a, (const value_t<DT>*)x);
                return;
            }
        }
        constexpr bool kMayBeWide = SRC != CIERA_SOURCE_ROWS || DT == CIERA_FP32;
        e = launch_after(wide && kMayBeWide ? quantize4_rows_kernel<DT, SRC, kMayBeWide> : quantize4_rows_kernel<DT, SRC, false>, grid, kFp4Threads, 0, s, a,
                         (const value_t<DT>*)x);
    });
    return e;
}

}  // namespace ciera

using namespace ciera;

extern "C" int ciera_fp4_quantize_rows(const ciera_fp4_rows* p, void* stream) {
    if (!p || p->rows > kMaxExtent || p->cols > kMaxExtent || p->x_rows > kMaxExtent) return CIERA_ERR_INVALID_ARG;
    if (p->source != CIERA_SOURCE_ROWS && p->source != CIERA_SOURCE_SWIGLU) return CIERA_ERR_INVALID_ARG;
    if (p->dtype != CIERA_BF16 && p->dtype != CIERA_FP32 && p->dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if (!p->rows) return CIERA_OK;
    const bool swiglu = p->source == CIERA_SOURCE_SWIGLU;
    const uint64_t width = swiglu ? 2 * p->cols : p->cols;
    if (p->cols < 1 || (p->x_rows && !p->x) || (p->x_rows > 1 && p->x_stride < width) ||
        (p->slot_of_row && (p->top_k < 1 || p->top_k > 32 || p->x_rows * p->top_k > kMaxExtent)) ||
        (p->starts && (p->n_experts < 1 || p->n_experts > 1024)) || ((swiglu || !p->slot_of_row) && p->x_rows < p->rows))
        return CIERA_ERR_INVALID_ARG;
    const int rc = operand4(p->q, p->q_stride, 0, p->scales, p->scales_stride, 0, 1, p->rows, p->cols);
    if (rc) return rc;
    if (!aligned_to(p->x, dtype_bytes(p->dtype)) || !aligned_to(p->slot_of_row, 4) || !aligned_to(p->starts, 4)) return CIERA_ERR_MISALIGNED;
    uint32_t each, chunks;
    const uint64_t units = rows_units(p->rows, p->cols, 1, &each, &chunks, swiglu ? kSwigluWarps : kRowWarps);
    if (units > kMaxExtent) return CIERA_ERR_UNSUPPORTED;
    const Rows4Args a{p->x_stride, 0, p->q_stride, 0, p->scales_stride, 0, p->x_rows, p->slot_of_row, p->starts, (uint32_t)p->rows,
                      (uint32_t)p->cols, (uint32_t)((p->cols + 255) / 256), (uint32_t)units, each, chunks, p->slot_of_row ? p->top_k : 1u, p->n_experts,
                      (uint32_t)p->x_rows, (uint8_t*)p->q, p->scales};
    const cudaError_t e = swiglu ? launch_rows4<CIERA_SOURCE_SWIGLU>(a, p->dtype, p->x, 1, (cudaStream_t)stream)
                                 : launch_rows4<CIERA_SOURCE_ROWS>(a, p->dtype, p->x, 1, (cudaStream_t)stream);
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}

extern "C" int ciera_fp4_quantize_matrices(const ciera_fp4_matrices* p, void* stream) {
    if (!p || p->rows > kMaxExtent || p->cols > kMaxExtent || p->matrices > 65535) return CIERA_ERR_INVALID_ARG;
    if (p->dtype != CIERA_BF16 && p->dtype != CIERA_FP32 && p->dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if ((p->q != nullptr) != (p->scales != nullptr) || (p->qt != nullptr) != (p->scales_t != nullptr) || (!p->q && !p->qt)) return CIERA_ERR_INVALID_ARG;
    if (!p->rows || !p->cols || !p->matrices) return CIERA_OK;
    if (!p->x || (p->rows > 1 && p->x_stride < p->cols)) return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(p->x, dtype_bytes(p->dtype))) return CIERA_ERR_MISALIGNED;
    if (p->q) {
        const int rc = operand4(p->q, p->q_stride, p->q_matrix_stride, p->scales, p->scales_stride, p->scales_matrix_stride, p->matrices, p->rows, p->cols);
        if (rc) return rc;
    }
    if (p->qt) {
        const int rc = operand4(p->qt, p->qt_stride, p->qt_matrix_stride, p->scales_t, p->scales_t_stride, p->scales_t_matrix_stride, p->matrices, p->cols, p->rows);
        if (rc) return rc;
    }
    uint32_t each, chunks;
    const uint64_t v = dtype_bytes(p->dtype), units = rows_units(p->rows, p->cols, p->matrices, &each, &chunks, kRowWarps), wide_cols = 256 / v;
    const uint64_t row_tiles = (p->rows + 127) / 128, col_tiles = (p->cols + wide_cols - 1) / wide_cols;
    if (units > kMaxExtent || row_tiles * col_tiles > kMaxExtent) return CIERA_ERR_UNSUPPORTED;
    cudaError_t e = cudaSuccess;
    if (p->q) {
        const Rows4Args a{p->x_stride, p->x_matrix_stride, p->q_stride, p->q_matrix_stride, p->scales_stride, p->scales_matrix_stride,
                          p->rows, nullptr, nullptr, (uint32_t)p->rows, (uint32_t)p->cols, (uint32_t)((p->cols + 255) / 256), (uint32_t)units, each, chunks, 1u, 0u,
                          (uint32_t)p->rows, (uint8_t*)p->q, p->scales};
        e = launch_rows4<CIERA_SOURCE_ROWS>(a, p->dtype, p->x, p->matrices, (cudaStream_t)stream);
        if (e != cudaSuccess) return record_cuda_error(e);
        count_launch();
    }
    if (p->qt) {
        const Turned4Args a{p->x_stride, p->x_matrix_stride, p->qt_stride, p->qt_matrix_stride, p->scales_t_stride, p->scales_t_matrix_stride,
                            (uint32_t)p->rows, (uint32_t)p->cols, (uint32_t)row_tiles, (uint32_t)col_tiles, (uint8_t*)p->qt, p->scales_t};
        const bool wide = !(((uint64_t)p->x | (p->rows > 1 ? p->x_stride * v : 0) | (p->matrices > 1 ? p->x_matrix_stride * v : 0) | p->cols * v) & 15);
        with_dtype(p->dtype, [&](auto dt) {
            constexpr int DT = decltype(dt)::value;
            e = launch_after(wide ? quantize4_turned_kernel<DT, true> : quantize4_turned_kernel<DT, false>,
                             dim3((uint32_t)(row_tiles * col_tiles), p->matrices), kFp4Threads, 0, (cudaStream_t)stream, a, (const value_t<DT>*)p->x);
        });
        if (e != cudaSuccess) return record_cuda_error(e);
        count_launch();
    }
    return CIERA_OK;
}

extern "C" int ciera_fp4_values(const ciera_fp4_value_args* p, void* stream) {
    if (!p || p->rows > kMaxExtent || p->cols > kMaxExtent || p->matrices > 65535) return CIERA_ERR_INVALID_ARG;
    if (p->dtype != CIERA_BF16 && p->dtype != CIERA_FP32 && p->dtype != CIERA_FP16) return CIERA_ERR_INVALID_ARG;
    if (!p->rows || !p->cols || !p->matrices) return CIERA_OK;
    if (!p->out || (p->rows > 1 && p->out_stride < p->cols)) return CIERA_ERR_INVALID_ARG;
    const int rc = operand4(p->q, p->q_stride, p->q_matrix_stride, p->scales, p->scales_stride, p->scales_matrix_stride, p->matrices, p->rows, p->cols);
    if (rc) return rc;
    const uint64_t v = dtype_bytes(p->dtype), units = warp_units(p->rows, p->cols);
    if (!aligned_to(p->out, v)) return CIERA_ERR_MISALIGNED;
    if (units > kMaxExtent) return CIERA_ERR_UNSUPPORTED;
    const Values4Args a{p->q_stride, p->q_matrix_stride, p->scales_stride, p->scales_matrix_stride, p->out_stride, p->out_matrix_stride,
                        (uint32_t)p->rows, (uint32_t)p->cols, (uint32_t)((p->cols + 255) / 256), (uint32_t)units, (const uint8_t*)p->q, p->scales};
    const bool wide = !(((uint64_t)p->out | (p->rows > 1 ? p->out_stride * v : 0) | (p->matrices > 1 ? p->out_matrix_stride * v : 0)) & 15);
    const dim3 grid((uint32_t)((units + kFp4Threads / 32 - 1) / (kFp4Threads / 32)), p->matrices);
    cudaError_t e = cudaSuccess;
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        e = launch_after(wide ? values4_kernel<DT, true> : values4_kernel<DT, false>, grid, kFp4Threads, 0, (cudaStream_t)stream, a, (value_t<DT>*)p->out);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    count_launch();
    return CIERA_OK;
}
