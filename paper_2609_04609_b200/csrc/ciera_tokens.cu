// A whole MoE layer for a few tokens.
//
// What it costs is reading the matrices of the experts that are reached, once: one token of 8 experts of 2048 x 1024 reads 50 MB
// in 8 bits and multiplies each weight once.  So a warp streams 16 rows of a matrix through 128 columns at a time, by
// asynchronous copies into a ring of its own (every lane reads what it has copied itself, so a warp waits for nobody), and has the
// 16-bit tensor cores multiply them, as rows of the first operand, with up to 8 tokens as columns of the second: both formats
// are exact in fp16, whose power of two comes after the sum over a block (or group) that shares it.  The tokens' values are made fp16
// below a power of two of their own for 128 values; fp32 ones in two parts.
//
// One kernel behind the router's, whose blocks all run at once (a cooperative launch), in two parts with a barrier between them:
//   up     a block takes tiles of 8 columns of the middle, 8 rows of the gate and 8 of up as the 16 rows of a warp, so that the sums
//          of both meet in one lane; its warps split the contraction, and several tiles' sums are added up in shared memory
//          together.  silu(g) * u goes to the workspace as fp16 below a power of two for its 8 columns.
//   down   a block takes 16 columns of the output and the warps split what they are summed over, experts and middle alike; a warp
//          adds each token's part to sums of its own, which are added up at the end in the order of the warps.
// A warp's copies go on from the one part's units to the other's, so the weights of the second are on their way (for one token nearly
// all of them) while the blocks wait for each other.
// Tokens of an expert are taken 8 at a time (16, with more than 8 tokens in all): a group.  Groups come in the order of the experts
// and of their slots, so a result does not depend on how warps run.
#include <type_traits>

#include "ciera_fp4.cuh"
#include "ciera_pipe.cuh"
#include "ciera_swiglu.cuh"

namespace ciera {

constexpr int kTokenThreads = 512, kTokenWarps = kTokenThreads / 32;
template <int BITS>
constexpr int kTokenRing = BITS == 8 ? 4 : 6;  // units of 16 rows x 128 columns that a warp has on their way, and the one it works on
constexpr uint32_t kTokenHead = 256;   // bytes of the workspace's counters
constexpr uint32_t kMaxSlots = CIERA_EXPERT_TOKENS_MAX * 32;
constexpr int kColumnPitch = 20;       // floats between columns of 16 sums: a warp's are in different banks
constexpr int kTokenPitch = 17;        // the same between tokens, which come in any order
constexpr uint32_t kLeastExponent = 16;  // of a power of two that values are taken below

struct Matrices {
    const uint8_t* q;
    const uint8_t* scales;
    uint64_t stride, matrix_stride, scales_stride, scales_matrix_stride;
};
struct TokensArgs {
    Matrices w1, w2;
    const int32_t* experts;
    const float* weights;
    uint64_t x_stride, out_stride;
    uint32_t* counters;  // blocks at the barrier, blocks that have left it: zero before and after
    int32_t* status;
    uint8_t* hidden;     // [places][parts][d_ff] fp16
    uint8_t* exponents;  // [places][d_ff / 8]
    uint32_t n_tokens, top_k, n_experts, d_model, d_ff;
    uint32_t splits, tiles;  // up: warps that share a tile, tiles of a block at a time
    int32_t x_wide;          // x may be read 16 bytes at a time
};

// The slots of the reached experts in the order of the experts, each at a place, and groups of up to `columns` of an expert's.
struct TokenLists {
    uint32_t group[kMaxSlots];  // expert << 16 | slots - 1 << 11 | first place
    float weight[kMaxSlots];
    uint8_t token[kMaxSlots];
    uint32_t warp_total[kTokenWarps];
    uint32_t groups;
};
struct ListScratch {
    uint32_t at[1024];  // slots of an expert; then their first place
    uint8_t count[kMaxSlots / 32 * 1024];  // [32 slots][expert]; n_experts apart
};
__device__ __forceinline__ uint32_t group_expert(uint32_t g) { return g >> 16; }
__device__ __forceinline__ uint32_t group_slots(uint32_t g) { return (g >> 11 & 31u) + 1; }
__device__ __forceinline__ uint32_t group_first(uint32_t g) { return g & 2047u; }

// By the whole block; ends with a barrier.
__device__ __forceinline__ void make_lists(TokenLists& l, ListScratch& s, const TokensArgs& a, uint32_t columns) {
    const uint32_t n = a.n_tokens * a.top_k, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.n_experts;
    if (n <= 32) {  // by one warp, a slot a lane
        if (warp == 0) {
            const int32_t id = lane < n ? __ldcg(a.experts + lane) : -1;
            const float w = lane < n ? __ldcg(a.weights + lane) : 0.f;
            const uint32_t e = (uint32_t)id < E ? (uint32_t)id : 0xffffu;
            uint32_t place = 0, rank = 0, count = 0, groups = 0;  // places before, before of the same expert, the expert's, groups before
            for (uint32_t i = 0; i < n; ++i) {
                const uint32_t o = __shfl_sync(~0u, e, i);
                place += o < e || (o == e && i < lane);
                rank += o == e && i < lane;
                count += o == e;
            }
            const bool first = rank % columns == 0 && e != 0xffffu;  // the lane makes a group
            for (uint32_t i = 0; i < n; ++i) groups += __shfl_sync(~0u, first ? place : ~0u, i) < place;
            if (e != 0xffffu) l.token[place] = (uint8_t)(lane / a.top_k), l.weight[place] = w;
            if (first) l.group[groups] = e << 16 | (min(columns, count - rank) - 1) << 11 | place;
            const uint32_t all = __popc(__ballot_sync(~0u, first));
            if (lane == 0) l.groups = all;
        }
        __syncthreads();
        return;
    }
    // slots of an expert are counted for each 32 neighbours, then over those before
    const uint32_t chunks = (n + 31) / 32;
    for (uint32_t i = tid; i < (chunks * E + 15) / 16; i += kTokenThreads) reinterpret_cast<uint4*>(s.count)[i] = make_uint4(0, 0, 0, 0);
    int32_t id[kMaxSlots / kTokenThreads];
#pragma unroll
    for (int j = 0; j < (int)(kMaxSlots / kTokenThreads); ++j) {
        const uint32_t i = j * kTokenThreads + tid;
        id[j] = i < n ? __ldcg(a.experts + i) : -1;
        if ((uint32_t)id[j] >= E) id[j] = -1;
    }
    __syncthreads();
    uint32_t rank[kMaxSlots / kTokenThreads];
#pragma unroll
    for (int j = 0; j < (int)(kMaxSlots / kTokenThreads); ++j) {
        const uint32_t chunk = j * kTokenWarps + warp;
        if (chunk >= chunks) break;
        const uint32_t same = __match_any_sync(~0u, id[j]);
        rank[j] = __popc(same & ((1u << lane) - 1));
        if (id[j] >= 0 && rank[j] == 0) s.count[chunk * E + id[j]] = (uint8_t)__popc(same);
    }
    __syncthreads();
    // places and groups before each expert, two experts a thread: slots in the low half, groups in the high one
    uint32_t c0 = 0, c1 = 0;
    if (2 * tid < E) {
        for (uint32_t i = 0; i < chunks; ++i) {
            c0 += s.count[i * E + 2 * tid];
            if (2 * tid + 1 < E) c1 += s.count[i * E + 2 * tid + 1];
        }
    }
    const uint32_t v0 = c0 | (c0 + columns - 1) / columns << 16, v1 = c1 | (c1 + columns - 1) / columns << 16;
    uint32_t sum = v0 + v1;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(~0u, sum, d);
        if (lane >= (uint32_t)d) sum += o;
    }
    if (lane == 31) l.warp_total[warp] = sum;
    __syncthreads();
    uint32_t base = 0;
    for (uint32_t w = 0; w < warp; ++w) base += l.warp_total[w];
    if (tid == kTokenThreads - 1) l.groups = (base + sum) >> 16;
    const uint32_t first[2] = {base + sum - v0 - v1, base + sum - v1}, count[2] = {c0, c1};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t e = 2 * tid + i, at = first[i] & 0xffffu;
        uint32_t g = first[i] >> 16;
        for (uint32_t c = 0; c < count[i]; c += columns, ++g) l.group[g] = e << 16 | (min(columns, count[i] - c) - 1) << 11 | (at + c);
        s.at[e] = at;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < (int)(kMaxSlots / kTokenThreads); ++j) {
        const uint32_t chunk = j * kTokenWarps + warp;
        if (chunk >= chunks) break;
        if (id[j] < 0) continue;
        uint32_t place = s.at[id[j]] + rank[j];
        for (uint32_t i = 0; i < chunk; ++i) place += s.count[i * E + id[j]];
        const uint32_t slot = j * kTokenThreads + tid;
        l.token[place] = (uint8_t)(slot / a.top_k);
        l.weight[place] = __ldcg(a.weights + slot);
    }
    __syncthreads();
}

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void from_e4m3x4(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(codes));
}

// A warp's unit: 16 rows of a matrix x 128 columns.  Lane (g, t) = (lane / 4, lane % 4) copies of rows g and g + 8
//   8 bits  columns 16 t ... and 64 + 16 t ..., 16 bytes each; block scales are read when they are needed
//   4 bits  columns 32 t ..., 16 bytes, a group; and the row's word of scales
// and has the tokens' values of its columns in this order, two to a register.  In 4 bits the lanes of a row exchange words first, so
// that all four have columns of one group at a time: 8 of them from 32 b + 8 t on, for b = 0 .. 3.
template <int BITS>
struct alignas(16) Unit;
template <>
struct alignas(16) Unit<8> {
    uint4 w[4][32];  // [row half * 2 + piece][lane]
};
template <>
struct alignas(16) Unit<4> {
    uint4 w[2][32];  // [row half][lane]
    uint32_t s[2][32];
};
template <int BITS>
__device__ __forceinline__ uint32_t fragment_column(int i, uint32_t t) {  // of the lane's value i, 0 .. 31
    return BITS == 8 ? (i >> 4) * 64 + t * 16 + (i & 15) : (i >> 3) * 32 + t * 8 + (i & 7);
}

// Where a lane's part of a unit comes from: rows lo + g and hi + g of matrix e (lo and hi - lo are multiples of 8), columns from
// 128 * kb on.
template <int BITS>
struct UnitSource {
    const uint8_t* a;
    const uint8_t* b;
    const uint8_t* sa;  // 4 bits: the scale words of rows g and hi - lo + g ...
    const uint8_t* sb;
    uint32_t lo;        // ... from which row lo's are this far

    __device__ __forceinline__ void point(const Matrices& m, uint32_t e, uint32_t row, uint32_t apart, uint32_t kb, int lane) {
        const uint32_t g = lane >> 2, t = lane & 3;
        a = m.q + e * m.matrix_stride + (uint64_t)(row + g) * m.stride + kb * (16 * BITS) + t * 16;
        b = a + (uint64_t)apart * m.stride;
        if constexpr (BITS == 4) {
            lo = row;
            sa = m.scales + e * m.scales_matrix_stride + (uint64_t)kb * kAtomBytes + g * 16;
            sb = apart == 8 ? sa + 128 : sa + (uint64_t)(apart >> 7) * m.scales_stride;  // (8: the same block of 32 rows)
        }
    }
    __device__ __forceinline__ void copy(uint32_t to, const Matrices& m, int lane) const {
        to += lane * 16;
        const auto copy16 = [](uint32_t dst, const uint8_t* p) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(p) : "memory");
        };
        copy16(to, a);
        if constexpr (BITS == 8) {
            copy16(to + 512, a + 64);
            copy16(to + 1024, b);
            copy16(to + 1536, b + 64);
        } else {
            copy16(to + 512, b);
            const uint64_t off = (uint64_t)(lo >> 7) * m.scales_stride + atom_word(lo);
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 1024 - lane * 12), "l"(sa + off) : "memory");
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 1152 - lane * 12), "l"(sb + off) : "memory");
        }
    }
};
// 8 bits: the scale of a row's block
__device__ __forceinline__ float block_scale(const Matrices& m, uint32_t e, uint32_t row, uint32_t kb) {
    return scale_value(__ldg(m.scales + e * m.scales_matrix_stride + (uint64_t)(row >> 7) * m.scales_stride + kb));
}

// The four words of a row's four lanes, turned: word j of lane t to word t of lane j.
__device__ __forceinline__ void turn_words(uint32_t (&w)[4], uint32_t t) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint32_t o = __shfl_xor_sync(~0u, t & 1 ? w[i] : w[i + 1], 1);
        if (t & 1) w[i] = o;
        else w[i + 1] = o;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t o = __shfl_xor_sync(~0u, t & 2 ? w[i] : w[i + 2], 2);
        if (t & 2) w[i] = o;
        else w[i + 2] = o;
    }
}

__device__ __forceinline__ uint4 read16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t read4(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// sums[nt] = the unit's rows times the columns of x, scales of the rows included: rows g, g + 8 of columns 2 t, 2 t + 1
template <int BITS, int NT, int P>
__device__ __forceinline__ void multiply_unit(uint32_t unit, const uint32_t (&x)[NT][P][16], float s_lo, float s_hi, float (&sums)[NT][4], int lane) {
    unit += lane * 16;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[nt][i] = 0.f;
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = read16(unit + 512 * i);
#pragma unroll
        for (int piece = 0; piece < 2; ++piece) {
            const uint32_t l[4] = {w[piece].x, w[piece].y, w[piece].z, w[piece].w}, h[4] = {w[2 + piece].x, w[2 + piece].y, w[2 + piece].z, w[2 + piece].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a0, a1, a2, a3;
                from_e4m3x4(l[j], a0, a2);
                from_e4m3x4(h[j], a1, a3);
                const int r = piece * 8 + 2 * j;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int p = 0; p < P; ++p) mma_16x8x16(sums[nt], a0, a1, a2, a3, x[nt][p][r], x[nt][p][r + 1]);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sums[nt][0] *= s_lo, sums[nt][1] *= s_lo, sums[nt][2] *= s_hi, sums[nt][3] *= s_hi;
    } else {
        const uint4 lo = read16(unit), hi = read16(unit + 512);
        const uint32_t sl = read4(unit + 1024 - lane * 12), sh = read4(unit + 1152 - lane * 12);
        uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, h[4] = {hi.x, hi.y, hi.z, hi.w};
        turn_words(l, lane & 3);
        turn_words(h, lane & 3);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            uint32_t a[4], c[4];
            from_e2m1x8(l[b], a);
            from_e2m1x8(h[b], c);
            const float fl = scale_value(sl >> (8 * b) & 255u), fh = scale_value(sh >> (8 * b) & 255u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    mma_16x8x16(part, a[0], c[0], a[1], c[1], x[nt][p][4 * b], x[nt][p][4 * b + 1]);
                    mma_16x8x16(part, a[2], c[2], a[3], c[3], x[nt][p][4 * b + 2], x[nt][p][4 * b + 3]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = i < 2 ? fl : fh;
                    sums[nt][i] = b == 0 ? part[i] * f : fmaf(part[i], f, sums[nt][i]);
                }
            }
        }
    }
}

// The biased exponent e of the power of two that values of these largest bits lie below (e = 255: not finite), what brings them
// below 2^15, and what takes it back.
__device__ __forceinline__ uint32_t exponent_of(uint32_t magnitude) { return max(magnitude >> 23, kLeastExponent); }
__device__ __forceinline__ float to_half_range(uint32_t e) { return __uint_as_float((268u - e) << 23); }
__device__ __forceinline__ float from_half_range(uint32_t e) { return __uint_as_float((e - 14u) << 23); }
// The rest of a value in that range behind its fp16 part.
__device__ __forceinline__ float rest_of(float v, __half h) {
    const float r = v - __half2float(h);
    return isfinite(r) ? r : 0.f;
}

// 128 values of a token (row) as a lane's column of the second operand, and what their sums are multiplied by.
template <int DT, int BITS, int P>
__device__ __forceinline__ float load_tokens(const value_t<DT>* __restrict__ row, bool there, bool wide, uint32_t (&x)[P][16], uint32_t t) {
    float v[32];
    if (there && wide) {
        constexpr int kEach = 16 / sizeof(value_t<DT>);
#pragma unroll
        for (int i = 0; i < 32; i += kEach) {
            float part[kEach];
            load_values<DT, kEach>(row + fragment_column<BITS>(i, t), part);
#pragma unroll
            for (int j = 0; j < kEach; ++j) v[i + j] = part[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = there ? ValueOf<DT>::get(row[fragment_column<BITS>(i, t)]) : 0.f;
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
    most = max(most, __shfl_xor_sync(~0u, most, 1));
    most = max(most, __shfl_xor_sync(~0u, most, 2));
    const uint32_t e = exponent_of(most);
    const float f = to_half_range(e);
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        const float lo = v[i] * f, hi = v[i + 1] * f;
        const __half2 h = __floats2half2_rn(lo, hi);
        x[0][i / 2] = *reinterpret_cast<const uint32_t*>(&h);
        if constexpr (P == 2) {
            const __half2 r = __floats2half2_rn(rest_of(lo, __low2half(h)), rest_of(hi, __high2half(h)));
            x[1][i / 2] = *reinterpret_cast<const uint32_t*>(&r);
        }
    }
    return from_half_range(e);
}

// The middle's values at a place, 128 of them, in a lane's order; scaled to the power of two of the largest.
template <int P>
struct HiddenPiece {
    uint4 v[P][4];
    uint4 e;
};
template <int BITS, int P>
__device__ __forceinline__ void read_hidden(HiddenPiece<P>& h, const TokensArgs& a, uint32_t place, uint32_t kb, bool there, uint32_t t) {
    if (!there) {
        h.e = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) h.v[p][i] = make_uint4(0, 0, 0, 0);
        return;
    }
    h.e = __ldcg(reinterpret_cast<const uint4*>(a.exponents + (uint64_t)place * (a.d_ff / 8) + kb * 16));
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const __half* from = reinterpret_cast<const __half*>(a.hidden) + ((uint64_t)place * P + p) * a.d_ff + kb * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) h.v[p][i] = __ldcg(reinterpret_cast<const uint4*>(from + fragment_column<BITS>(8 * i, t)));
    }
}
// 2^-n as fp16, twice; 0 where there is none
__device__ __forceinline__ uint32_t half_power(uint32_t n) {
    const uint32_t h = n < 15 ? (15 - n) << 10 : n < 25 ? 1u << (24 - n) : 0u;
    return h | h << 16;
}
template <int BITS, int P>
__device__ __forceinline__ float settle_hidden(const HiddenPiece<P>& h, uint32_t (&x)[P][16], uint32_t t) {
    uint32_t m = __vmaxu4(__vmaxu4(h.e.x, h.e.y), __vmaxu4(h.e.z, h.e.w));
    m = __vmaxu4(m, m >> 16);
    const uint32_t e = max(max(m & 255u, m >> 8 & 255u), kLeastExponent);
    const uint32_t word[4] = {h.e.x, h.e.y, h.e.z, h.e.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t own;  // the exponent of the lane's values 8 i .. 8 i + 7
        if (BITS == 8) own = ((t & 2 ? word[(i >> 1) * 2 + 1] : word[(i >> 1) * 2]) >> ((t & 1) * 16 + (i & 1) * 8)) & 255u;
        else own = word[i] >> (8 * t) & 255u;
        const uint32_t f = half_power(e - own);
        const __half2 factor = *reinterpret_cast<const __half2*>(&f);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const uint32_t v[4] = {h.v[p][i].x, h.v[p][i].y, h.v[p][i].z, h.v[p][i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&v[j]), factor);
                x[p][4 * i + j] = *reinterpret_cast<const uint32_t*>(&y);
            }
        }
    }
    return from_half_range(e);
}

template <int BITS>
struct TokensSmem {
    Unit<BITS> ring[kTokenWarps][kTokenRing<BITS>];
    TokenLists lists;
    int stop;
    // up: [rounds of a batch][warp][column][kColumnPitch]; down: [warp][token][kTokenPitch]
    __align__(16) float sums[];
};
// rounds of tiles whose sums are added up together, and what they need
template <int NT>
constexpr uint32_t kBatch = NT == 1 ? 8 : 4;
template <int NT>
constexpr uint32_t kBatchFloats = kBatch<NT> * kTokenWarps * NT * 8 * kColumnPitch;

// All blocks have come here, and what they wrote before can be read (past the first-level cache).  false: the wait ran out.
__device__ __forceinline__ bool all_blocks(const TokensArgs& a, int& stop) {
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t seen, polls = 0;
        __threadfence();
        atomicAdd(a.counters, 1u);
        do {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(a.counters) : "memory");
        } while (seen < gridDim.x && ++polls < kMaxPolls);
        stop = seen < gridDim.x;
        if (stop && a.status) atomicCAS(a.status, 0, (int32_t)CIERA_ERR_TIMEOUT);
        // the last one to leave sets both counters back
        if (!stop && atomicAdd(a.counters + 1, 1u) == gridDim.x - 1) {
            a.counters[0] = 0;
            a.counters[1] = 0;
        }
    }
    __syncthreads();
    return !stop;
}

template <int DT, int BITS, int NT>
__global__ void __launch_bounds__(kTokenThreads, 1) tokens_kernel(const TokensArgs a, const value_t<DT>* __restrict__ x_, value_t<DT>* __restrict__ out) {
    constexpr int P = DT == CIERA_FP32 ? 2 : 1, R = kTokenRing<BITS>;
    extern __shared__ __align__(16) uint8_t tokens_smem[];
    TokensSmem<BITS>& sm = *reinterpret_cast<TokensSmem<BITS>*>(tokens_smem);
    static_assert(sizeof(ListScratch) <= sizeof(sm.ring), "the lists are made where the ring will be");
    pdl_wait();
    make_lists(sm.lists, *reinterpret_cast<ListScratch*>(&sm.ring), a, NT * 8);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t g = lane >> 2, t = lane & 3;
    // the warp's ring: the next unit to be copied and to be worked on
    const uint32_t ring = smem_u32(sm.ring[warp]), ring_end = ring + sizeof(sm.ring[warp]);
    uint32_t c_at = ring, at = ring;
    const auto advance = [&](uint32_t& p) {
        p += sizeof(Unit<BITS>);
        if (p == ring_end) p = ring;
    };

    // up: tiles of 8 columns of the middle, in the order of the groups; a block has neighbouring ones, `tiles` at a time
    const uint32_t kb_up = a.d_model / 128, across = a.d_ff / 8;
    const uint64_t all = (uint64_t)sm.lists.groups * across;
    const uint32_t from = (uint32_t)(all * blockIdx.x / gridDim.x), to = (uint32_t)(all * (blockIdx.x + 1) / gridDim.x);
    const uint32_t mine = warp / a.splits, split = warp - mine * a.splits;  // the warp's tile of those, its part of the contraction
    const uint32_t rounds = (to - from + a.tiles - 1) / a.tiles;
    const uint32_t own = mine < a.tiles ? to : 0;  // the warp's tiles end here
    const uint32_t first_group = from / across, first_tile = from - first_group * across;
    // down: 16 columns of the output, everything that they are summed over
    const uint32_t kb_down = a.d_ff / 128, units = sm.lists.groups * kb_down;
    const uint32_t w_group = warp / kb_down, w_kb = warp - w_group * kb_down;

    // Copies go in runs, in which the source moves on by the same step: the warp's tiles of one group, or, where a warp has more than
    // one part of a tile's contraction, those; then single units of the second matrices.
    UnitSource<BITS> src;
    const bool by_tile = kb_up <= a.splits;
    uint32_t c_task = from + mine, c_group = first_group, c_tile = first_tile + mine, c_left = 0;
    uint32_t d_row = blockIdx.x * 16, d_unit = warp, d_group = w_group, d_kb = w_kb;
    bool up = true;
    const uint64_t a_step = by_tile ? (uint64_t)a.tiles * 8 * a.w1.stride : a.splits * (16 * BITS);
    const auto next_run = [&]() {
        if (up && c_task < own) {
            while (c_tile >= across) c_tile -= across, ++c_group;
            src.point(a.w1, group_expert(sm.lists.group[c_group]), c_tile * 8, a.d_ff, split, lane);
            if (by_tile) {
                c_left = (min(across - c_tile, own - c_task) + a.tiles - 1) / a.tiles;
                c_task += c_left * a.tiles;
                c_tile += c_left * a.tiles;
            } else {
                c_left = (kb_up - split + a.splits - 1) / a.splits;
                c_task += a.tiles;
                c_tile += a.tiles;
            }
            return;
        }
        up = false;
        if (d_unit >= units) {
            d_unit = warp, d_group = w_group, d_kb = w_kb;
            d_row += gridDim.x * 16;
        }
        if (d_row < a.d_model && d_unit < units) {
            src.point(a.w2, group_expert(sm.lists.group[d_group]), d_row, 8, d_kb, lane);
            c_left = 1;
            d_unit += kTokenWarps;
            d_kb += kTokenWarps;
            while (d_kb >= kb_down) d_kb -= kb_down, ++d_group;
        }
    };
    next_run();
    const auto copy = [&]() {
        if (c_left) {
            src.copy(c_at, up ? a.w1 : a.w2, lane);
            src.a += a_step;
            src.b += a_step;
            if (BITS == 4) {
                if (by_tile) src.lo += a.tiles * 8;
                else src.sa += a.splits * kAtomBytes, src.sb += a.splits * kAtomBytes;
            }
            if (--c_left == 0) next_run();
        }
        advance(c_at);
        cp_async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < R - 1; ++i) copy();

    {
        uint32_t task = from + mine, group = first_group, tile = first_tile + mine, loaded_group = ~0u, loaded_kb = ~0u, scaled = ~0u;
        uint32_t packed = 0, slots = 0;
        uint32_t xf[NT][P][16];
        float scale[NT][2], s_lo = 1.f, s_hi = 1.f;
        uint32_t b_group = first_group, b_tile = first_tile;  // of the batch
        for (uint32_t r0 = 0; r0 < rounds; r0 += kBatch<NT>) {
            const uint32_t batch = min(kBatch<NT>, rounds - r0);
            float* put = sm.sums + (warp * NT * 8 + 2 * t) * kColumnPitch + g;
            for (uint32_t r = 0; r < batch && task < own; ++r) {
                while (tile >= across) tile -= across, ++group;
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nt][i] = 0.f;
                for (uint32_t kb = split; kb < kb_up; kb += a.splits) {
                    const bool other = group != loaded_group || kb != loaded_kb;
                    if (other) {
                        loaded_group = group, loaded_kb = kb;
                        packed = sm.lists.group[group];
                        slots = group_slots(packed);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint32_t c = nt * 8 + g;
                            const uint32_t token = c < slots ? sm.lists.token[group_first(packed) + c] : 0u;
                            const float f = load_tokens<DT, BITS, P>(x_ + token * a.x_stride + kb * 128, c < slots, a.x_wide, xf[nt], t);
                            scale[nt][0] = __shfl_sync(~0u, f, 8 * t);
                            scale[nt][1] = __shfl_sync(~0u, f, 8 * t + 4);
                        }
                    }
                    if (BITS == 8 && (other || tile >> 4 != scaled)) {
                        scaled = tile >> 4;
                        s_lo = block_scale(a.w1, group_expert(packed), tile * 8, kb);
                        s_hi = block_scale(a.w1, group_expert(packed), a.d_ff + tile * 8, kb);
                    }
                    cp_async_wait<R - 2>();
                    float sums[NT][4];
                    multiply_unit<BITS, NT, P>(at, xf, s_lo, s_hi, sums, lane);
                    advance(at);
                    copy();
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[nt][j] = fmaf(sums[nt][j], scale[nt][j & 1], acc[nt][j]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float* p = put + nt * 8 * kColumnPitch;
                    if (nt * 8 + 2 * t < slots) p[0] = acc[nt][0], p[8] = acc[nt][2];
                    if (nt * 8 + 2 * t + 1 < slots) p[kColumnPitch] = acc[nt][1], p[kColumnPitch + 8] = acc[nt][3];
                }
                put += kTokenWarps * NT * 8 * kColumnPitch;
                task += a.tiles;
                tile += a.tiles;
            }
            __syncthreads();
            // A warp adds up a column of 8 gates and 8 ups, four lanes a sum: column warp % (8 NT) of every (2 / NT)th tile.
            const uint32_t column = warp % (NT * 8), of_batch = min(batch * a.tiles, to - from - r0 * a.tiles);
            uint32_t c_in = b_tile + warp / (NT * 8), c_of = b_group;
            for (uint32_t which = warp / (NT * 8), r = 0, first = 0; which < of_batch; which += 2 / NT, c_in += 2 / NT) {
                while (c_in >= across) c_in -= across, ++c_of;
                const uint32_t p = sm.lists.group[c_of];
                if (column >= group_slots(p)) continue;
                if (a.tiles == 1) r = which;
                else r = which / a.tiles, first = (which - r * a.tiles) * a.splits;
                const float* part = sm.sums + ((r * kTokenWarps + first + (lane >> 3)) * NT * 8 + column) * kColumnPitch + (lane & 7);
                float gate = 0.f, up_ = 0.f;
#pragma unroll
                for (int s = 0; s < kTokenWarps; s += 4)
                    if (s + (lane >> 3) < a.splits) {
                        gate += part[s * NT * 8 * kColumnPitch];
                        up_ += part[s * NT * 8 * kColumnPitch + 8];
                    }
#pragma unroll
                for (int d = 8; d < 32; d <<= 1) {
                    gate += __shfl_xor_sync(~0u, gate, d);
                    up_ += __shfl_xor_sync(~0u, up_, d);
                }
                float v = swiglu32(gate, up_);
                if (gate < kLowestGate) v = (float)((double)gate / (1.0 + exp(-(double)gate)) * (double)up_);
                uint32_t most = __float_as_uint(v) & 0x7fffffffu;
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) most = max(most, __shfl_xor_sync(~0u, most, d));
                const uint32_t e = exponent_of(most), place = group_first(p) + column;
                if (lane < 8) {
                    v *= to_half_range(e);
                    __half* h = reinterpret_cast<__half*>(a.hidden) + (uint64_t)place * P * a.d_ff + c_in * 8 + lane;
                    const __half hi = __float2half_rn(v);
                    h[0] = hi;
                    if (P == 2) h[a.d_ff] = __float2half_rn(rest_of(v, hi));
                    if (lane == 0) a.exponents[(uint64_t)place * across + c_in] = (uint8_t)e;
                }
            }
            b_tile += batch * a.tiles;
            while (b_tile >= across) b_tile -= across, ++b_group;
            if (r0 + batch < rounds) __syncthreads();
        }
    }
    if (!all_blocks(a, sm.stop)) {
        cp_async_wait_all();
        return;
    }

    float* sums = sm.sums + warp * a.n_tokens * kTokenPitch;
    HiddenPiece<P> piece[NT];
    float s_next = 1.f;
    uint32_t group = w_group, kb = w_kb;  // of `unit`
    const auto read = [&](uint32_t row) {
        const uint32_t packed = sm.lists.group[group], slots = group_slots(packed);
        if (BITS == 8) s_next = block_scale(a.w2, group_expert(packed), row, kb);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) read_hidden<BITS, P>(piece[nt], a, group_first(packed) + nt * 8 + g, kb, nt * 8 + g < slots, t);
    };
    for (uint32_t row = blockIdx.x * 16; row < a.d_model; row += gridDim.x * 16) {
        group = w_group, kb = w_kb;
        if ((uint32_t)warp < units) read(row);
        for (uint32_t i = lane; i < a.n_tokens * kTokenPitch; i += 32) sums[i] = 0.f;
        __syncwarp();
        for (uint32_t unit = warp; unit < units; unit += kTokenWarps) {
            const uint32_t packed = sm.lists.group[group], slots = group_slots(packed);
            uint32_t xf[NT][P][16];
            float f[NT];
            const float s = s_next;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) f[nt] = settle_hidden<BITS, P>(piece[nt], xf[nt], t);
            kb += kTokenWarps;
            while (kb >= kb_down) kb -= kb_down, ++group;
            if (unit + kTokenWarps < units) read(row);
            cp_async_wait<R - 2>();
            float part[NT][4];
            multiply_unit<BITS, NT, P>(at, xf, s, s, part, lane);
            advance(at);
            copy();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t c = nt * 8 + 2 * t + i;
                    const float fc = __shfl_sync(~0u, f[nt], 8 * t + 4 * i);
                    if (c >= slots) continue;
                    const uint32_t place = group_first(packed) + c;
                    const float w = sm.lists.weight[place];
                    float* to = sums + sm.lists.token[place] * kTokenPitch + g;
                    to[0] = fmaf(part[nt][i] * fc, w, to[0]);
                    to[8] = fmaf(part[nt][2 + i] * fc, w, to[8]);
                }
            __syncwarp();
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < a.n_tokens * 16; i += kTokenThreads) {
            const uint32_t token = i / 16, r = i % 16;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kTokenWarps; ++w) v += sm.sums[((uint32_t)w * a.n_tokens + token) * kTokenPitch + r];
            out[token * a.out_stride + row + r] = ValueOf<DT>::put(v);
        }
        if (row + gridDim.x * 16 < a.d_model) __syncthreads();
    }
    cp_async_wait_all();
}

template <class K>
static cudaError_t allow_shared(K kernel, size_t bytes, std::atomic<uint64_t>& allowed) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (allowed.load(std::memory_order_relaxed) >> dev & 1)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

template <int DT, int BITS, int NT>
static cudaError_t launch_tokens(const TokensArgs& a, const void* x, void* out, uint32_t sms, cudaStream_t s) {
    static std::atomic<uint64_t> allowed{0};
    constexpr uint64_t most = 4ull * kTokenWarps * CIERA_EXPERT_TOKENS_MAX * kTokenPitch;
    static_assert(sizeof(TokensSmem<BITS>) + (most > 4 * kBatchFloats<NT> ? most : 4 * kBatchFloats<NT>) <= 227 * 1024, "more than a block may have");
    const uint64_t down = 4ull * kTokenWarps * a.n_tokens * kTokenPitch, up = 4 * kBatchFloats<NT>;
    auto kernel = tokens_kernel<DT, BITS, NT>;
    cudaError_t e = allow_shared(kernel, sizeof(TokensSmem<BITS>) + (most > up ? most : up), allowed);
    if (e != cudaSuccess) return e;
    // no more blocks than have work in one of the parts
    const uint64_t tasks = (uint64_t)a.n_tokens * a.top_k * (a.d_ff / 8), rows = a.d_model / 16, work = tasks > rows ? tasks : rows;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)(work < sms ? work : sms));
    cfg.blockDim = dim3(kTokenThreads);
    cfg.dynamicSmemBytes = sizeof(TokensSmem<BITS>) + (down > up ? down : up);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, kernel, a, (const value_t<DT>*)x, (value_t<DT>*)out);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace ciera

using namespace ciera;

extern "C" size_t ciera_expert_tokens_workspace_bytes(uint32_t n_tokens, uint32_t top_k, uint32_t d_ff) {
    // silu(g) * u of every slot in at most two parts of fp16, and an exponent for 8 of them
    const uint64_t values = (uint64_t)n_tokens * top_k * d_ff;
    return kTokenHead + 4 * values + (values / 8 + 15) / 16 * 16;
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
        return (int)CIERA_OK;
    };
    if (t) {
        int rc = weights(p->w1, p->w1_stride, p->w1_matrix_stride, p->w1_scales, p->w1_scales_stride, p->w1_scales_matrix_stride, 2 * f, d);
        if (!rc) rc = weights(p->w2, p->w2_stride, p->w2_matrix_stride, p->w2_scales, p->w2_scales_stride, p->w2_scales_matrix_stride, d, f);
        if (rc) return rc;
        if (!aligned_to(p->x, dtype_bytes(p->dtype)) || !aligned_to(p->out, dtype_bytes(p->dtype)) || !aligned_to(p->workspace, 16) ||
            !aligned_to(p->status, 4))
            return CIERA_ERR_MISALIGNED;
        if (p->workspace_bytes < ciera_expert_tokens_workspace_bytes(p->n_tokens, p->route.top_k, p->d_ff)) return CIERA_ERR_CAPACITY;
    }
    const int rc = ciera_route(&p->route, p->logits_dtype, p->logits, t, p->logits_stride, p->bias, p->experts, p->weights, stream);
    if (rc || !t) return rc;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    // warps that share a tile's contraction, at most one 128 columns each, and the tiles that a block then has at a time
    const uint32_t kb = (uint32_t)(d / 128), splits = kb < kTokenWarps ? kb : kTokenWarps, tiles = kTokenWarps / splits;
    const uint64_t values = t * p->route.top_k * f, v = dtype_bytes(p->dtype);
    const bool x_wide = !(((uint64_t)p->x | (t > 1 ? p->x_stride * v : 0)) & 15);
    uint8_t* room = (uint8_t*)p->workspace + kTokenHead;
    const TokensArgs a{{(const uint8_t*)p->w1, p->w1_scales, p->w1_stride, p->w1_matrix_stride, p->w1_scales_stride, p->w1_scales_matrix_stride},
                       {(const uint8_t*)p->w2, p->w2_scales, p->w2_stride, p->w2_matrix_stride, p->w2_scales_stride, p->w2_scales_matrix_stride},
                       p->experts, p->weights, p->x_stride, p->out_stride, (uint32_t*)p->workspace, p->status, room, room + 4 * values,
                       (uint32_t)t, p->route.top_k, p->route.n_experts, (uint32_t)d, (uint32_t)f, splits, tiles, x_wide};
    with_dtype(p->dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto go = [&](auto bits, auto nt) {
            e = launch_tokens<DT, decltype(bits)::value, decltype(nt)::value>(a, p->x, p->out, (uint32_t)sms, (cudaStream_t)stream);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 8> eight;
        const std::integral_constant<int, 4> bits4;
        if (four) t <= 8 ? go(bits4, one) : go(bits4, two);
        else t <= 8 ? go(eight, one) : go(eight, two);
    });
    if (e != cudaSuccess) return record_cuda_error(e);
    return CIERA_OK;
}
