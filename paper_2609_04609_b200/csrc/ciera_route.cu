// Routing of tokens to experts, and its gradient.
//
// The choice is that of 64-bit arithmetic.  It is made in 32 bits (route_kernel) and looked over: where two values in the
// order of choice, or the groups on either side of the last one kept, are nearer to each other than 32 bits can tell, and do not
// come from the same logit and bias, the token is done again in 64 bits (route_exact).
//
// L lanes take a token and go through its row, each with a sorted list of the largest values in registers, as single words that
// hold the place beside the value (with groups, through shared memory, for their values come first).  The lists are merged,
// and the few that are left are compared as they are.  16384 tokens of 256 experts in 8 groups take 24 us, 510 instructions a token:
// one wave of about 14 warps an SM, each from its loads to its stores in steps that depend on each other (a third of the issue
// slots is used), and 5 us for the tokens that are done again.  (The k largest picked one by one by the whole warp: 43 us, 1600
// instructions a token.)
#include <math.h>

#include <type_traits>

#include "ciera_numeric.cuh"

namespace ciera {

constexpr int kRouteWarps = 4;

struct RouteArgs {
    uint32_t n_experts, top_k, n_groups, top_groups, group_best, group_size;
    int32_t sigmoid, renormalise;
    float scale;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, d));
    return v;
}

// a logit as it counts: closed (-inf) or finite, and one zero (its bits are compared)
__device__ __forceinline__ float open_logit(float x) { return isnan(x) ? -INFINITY : fminf(x, 3.402823466e38f) + 0.f; }

// The lane's EPL logits; whole: one access for up to 16 bytes of them.
template <int DT, int EPL>
__device__ __forceinline__ void load_logits(const value_t<DT>* row, uint32_t E, bool whole, int lane, float (&x)[EPL]) {
    const uint32_t e0 = lane * EPL;
    if (whole && e0 + EPL <= E) {
        load_values<DT, EPL>(row + e0, x);
    } else {
#pragma unroll
        for (int j = 0; j < EPL; ++j) x[j] = e0 + j < E ? ValueOf<DT>::get(row[e0 + j]) : -INFINITY;
    }
}

// 64-bit numbers as unsigned integers of the same order, which compare in a fraction of the time; 0 for -inf and NaN
__device__ __forceinline__ unsigned long long ordered64(double v) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(v == 0.0 ? 0.0 : v);
    return v > -INFINITY ? (u >> 63 ? ~u : u | 1ull << 63) : 0ull;
}
__device__ __forceinline__ double unordered64(unsigned long long u) {
    return u ? __longlong_as_double((long long)(u >> 63 ? u & ~(1ull << 63) : ~u)) : -INFINITY;
}

// 1 / d for d from 1 to infinity, by Newton's iteration r <- r + r (1 - d r) from 24 bits: 48, then all 53 but the last.  (A
// division of 64 bits is a call, and as many calls as a lane has experts are done one behind the other.)
__device__ __forceinline__ double reciprocal64(double d) {
    double r = (double)__fdividef(1.f, (float)d);
    r = fma(r, fma(-d, r, 1.0), r);
    r = fma(r, fma(-d, r, 1.0), r);
    return d < 1e30 ? r : 1.0 / d;
}

// One token's choice in 64 bits.  c: n_experts words of 64 bits of the warp's own in shared memory.  What a batch waits for when
// it has such a token, so with all the parallelism there is: a lane's experts side by side, several lanes to a group.
template <int DT, int EPL>
__device__ __noinline__ void route_exact(const value_t<DT>* row, const RouteArgs a, const float* __restrict__ bias, unsigned long long* c,
                                         int32_t* __restrict__ experts, float* __restrict__ weights) {
    const uint32_t E = a.n_experts, lane = threadIdx.x & 31, e0 = lane * EPL;
    float x[EPL];
    load_logits<DT, EPL>(row, E, false, (int)lane, x);
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        x[j] = open_logit(x[j]);
        m = fmaxf(m, x[j]);
    }
    m = warp_max(m);
    double s[EPL], total = 0.0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        s[j] = 0.0;
        if (x[j] == -INFINITY) continue;
        s[j] = exp(a.sigmoid ? -(double)x[j] : (double)x[j] - (double)m);
        total += s[j];
    }
    if (!a.sigmoid) total = warp_sum(total);
    const double per_total = 1.0 / total;
    unsigned long long key[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        key[j] = 0ull;
        if (x[j] == -INFINITY) continue;
        s[j] = a.sigmoid ? reciprocal64(1.0 + s[j]) : s[j] * per_total;
        key[j] = ordered64(s[j] + (bias ? (double)bias[e0 + j] : 0.0));
    }
    if (a.top_groups < a.n_groups) {
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (e0 + j < E) c[e0 + j] = key[j];
        __syncwarp();
        uint32_t per = 32;  // lanes of a group
        while (per * a.n_groups > 32) per /= 2;
        const uint32_t g = lane / per;
        unsigned long long most = 0ull, second = 0ull;
        const auto see = [&](unsigned long long y) {
            second = max(second, min(most, y));
            most = max(most, y);
        };
        if (g < a.n_groups)
            for (uint32_t i = lane % per; i < a.group_size; i += per) see(c[g * a.group_size + i]);
        for (uint32_t d = 1; d < per; d *= 2) {
            const unsigned long long om = __shfl_xor_sync(~0u, most, d), os = __shfl_xor_sync(~0u, second, d);
            see(om);
            second = max(second, os);
        }
        const unsigned long long value = a.group_best > 1 && second ? ordered64(unordered64(most) + unordered64(second)) : most;
        uint32_t rank = 0;
        for (uint32_t i = 0; i < a.n_groups; ++i) {
            const unsigned long long o = __shfl_sync(~0u, value, i * per);
            rank += o > value || (o == value && i < g);
        }
        const uint32_t keep = __ballot_sync(~0u, value && rank < a.top_groups);
        const float per_size = __fdividef(1.f, (float)a.group_size);
#pragma unroll
        for (int j = 0; j < EPL; ++j) {  // (of places below 1024 the quotient is exact: a half is further from a whole than 2^-12)
            const uint32_t g_of = (uint32_t)(((float)(e0 + j) + 0.5f) * per_size);
            if (e0 + j < E && !(keep >> (g_of * per) & 1u)) key[j] = 0ull;
        }
        __syncwarp();
    }
    // lane i ends up with choice i: the largest, by the upper half first
    int chosen = -1;
    double ws = 0.0, sum = 0.0;
    for (uint32_t r = 0; r < a.top_k; ++r) {
        unsigned long long best = 0ull;
        double bs = 0.0;
        int be = 0;
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (key[j] > best) best = key[j], be = (int)e0 + j, bs = s[j];
        const uint32_t up = __reduce_max_sync(~0u, (uint32_t)(best >> 32));
        if (!up) break;
        const uint32_t down = __reduce_max_sync(~0u, (uint32_t)(best >> 32) == up ? (uint32_t)best : 0u);
        const int w = __ffs(__ballot_sync(~0u, (uint32_t)(best >> 32) == up && (uint32_t)best == down)) - 1;  // (the lowest of equal ones)
        const double taken = __shfl_sync(~0u, bs, w);
        const int e = __shfl_sync(~0u, be, w);
        if (lane == r) chosen = e, ws = taken;
        sum += taken;
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if ((int)e0 + j == e) key[j] = 0ull;
    }
    if (lane < a.top_k) {
        if (a.renormalise) ws = sum > 0.0 ? ws / sum : 0.0;
        experts[lane] = chosen;
        weights[lane] = (float)(ws * (double)a.scale);
    }
    __syncwarp();
}

// a float as an unsigned integer of the same order; every number is above 0
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t b = __float_as_uint(f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

__device__ __forceinline__ float sigmoid_of(float x) { return __fdividef(1.f, 1.f + expf(-x)); }

// How far two values have to be apart for 32 bits to tell them.  A score by sigmoid is off by less than 3e-7: the exponential by two
// steps of itself (times s (1 - s), at most a quarter), the sum by half a step, the reciprocal by two, and c by half a step of
// itself.  Softmax's by less than 5e-6 of itself, with what all its scores share, a sum of up to 1024 terms over 4 to 32 lanes: up to
// 64 additions in a lane, half a step each (3.8e-6), and what a term is off by; two of them by 5e-6 of the larger and a step of each.
constexpr float kUnsureSigmoid = 4e-7f, kUnsureSoftmax = 6e-6f;
// two values c whose scores are at most s: of both, for a bias may put a large score beside a small one
__device__ __forceinline__ float unsure_values(bool sigmoid, float s, float c) {
    return sigmoid ? 2.f * kUnsureSigmoid + 2e-7f * fabsf(c) : kUnsureSoftmax * (s + fabsf(c));
}
// two groups' values, of up to two scores each, which are at most s where there is a bias
__device__ __forceinline__ float unsure_groups(bool sigmoid, bool bias, float s, float a, float b) {
    const float size = fabsf(a) + fabsf(b);
    return sigmoid ? 4.f * kUnsureSigmoid + 3e-7f * size : kUnsureSoftmax * (size + (bias ? 4.f * s : 0.f));
}

// Chosen scores whose sum is below this are divided by it in 64 bits: their quotients are ordinary numbers, but some of them, or all,
// are no normal 32-bit ones.
constexpr float kSmallSum = 1e-10f;

constexpr uint32_t kClosed = 0x007fffffu;  // ordered(-inf): words up to here are of closed experts

// The lane's words in falling order.
template <int EPL>
__device__ __forceinline__ void sort_words(uint32_t (&key)[EPL]) {
#pragma unroll
    for (int run = 2; run <= EPL; run *= 2)
#pragma unroll
        for (int step = run / 2; step; step /= 2)
#pragma unroll
            for (int i = 0; i < EPL; ++i)
                if (!(i & step)) {
                    const uint32_t hi = max(key[i], key[i + step]), lo = min(key[i], key[i + step]);
                    const bool falling = !(i & run) || run == EPL;
                    key[i] = falling ? hi : lo;
                    key[i + step] = falling ? lo : hi;
                }
}

// Few tokens: a warp for each, which picks the largest one by one.
template <int DT, int EPL>
__global__ void __launch_bounds__(kRouteWarps * 32)
    route_few_kernel(const RouteArgs a, const value_t<DT>* __restrict__ logits, uint64_t n_tokens, uint64_t stride, int whole,
                     const float* __restrict__ bias, int32_t* __restrict__ experts, float* __restrict__ weights) {
    extern __shared__ __align__(16) float route_smem[];
    __shared__ int chosen[kRouteWarps][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t E = a.n_experts, e0 = lane * EPL;
    float* scratch = route_smem + warp * 2 * E;
    const uint64_t t = (uint64_t)blockIdx.x * kRouteWarps + warp;
    if (t >= n_tokens) return;
    const bool grouped = a.top_groups < a.n_groups, scored = bias || grouped;
    const value_t<DT>* row = logits + t * stride;
    float x[EPL], c[EPL], m = 0.f, inv = 1.f;
    load_logits<DT, EPL>(row, E, whole, lane, x);
#pragma unroll
    for (int j = 0; j < EPL; ++j) x[j] = open_logit(x[j]);
    if (!a.sigmoid) {
        m = x[0];
#pragma unroll
        for (int j = 1; j < EPL; ++j) m = fmaxf(m, x[j]);
        m = unordered(__reduce_max_sync(~0u, ordered(m)));
        if (m == -INFINITY) m = 0.f;  // nothing is open
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < EPL; ++j) sum += c[j] = expf(x[j] - m);
        sum = warp_sum(sum);
        inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
    }
    // what the choice goes by: the logits where there is no bias (scores rise with them), else s + b
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        if (!scored || x[j] == -INFINITY) c[j] = x[j];
        else c[j] = (a.sigmoid ? sigmoid_of(x[j]) : c[j] * inv) + (bias ? bias[e0 + j] : 0.f);
        if (isnan(c[j])) c[j] = -INFINITY;
    }
    bool sure = a.top_k < 32;  // (there is no lane for the first that is not chosen)
    if (grouped) {
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (e0 + j < E) scratch[e0 + j] = c[j];
        __syncwarp();
        uint32_t per = 32;  // lanes of a group
        while (per * a.n_groups > 32) per /= 2;
        const uint32_t g = lane / per;
        float most = -INFINITY, second = -INFINITY;
        if (g < a.n_groups)
            for (uint32_t i = lane % per; i < a.group_size; i += per) {
                const float y = scratch[g * a.group_size + i];
                second = fmaxf(second, fminf(most, y));
                most = fmaxf(most, y);
            }
        for (uint32_t d = 1; d < per; d *= 2) {
            const float om = __shfl_xor_sync(~0u, most, d), os = __shfl_xor_sync(~0u, second, d);
            second = fmaxf(fmaxf(second, os), fminf(most, om));
            most = fmaxf(most, om);
        }
        const float value = a.group_best > 1 && second > -INFINITY ? most + second : most;
        uint32_t rank = 0;
        for (uint32_t i = 0; i < a.n_groups; ++i) {
            const float o = __shfl_sync(~0u, value, i * per);
            rank += o > value || (o == value && i < g);
        }
        const bool open = g < a.n_groups && most > -INFINITY, stays = open && rank < a.top_groups;
        if (open && value == -INFINITY) sure = false;  // (two open experts whose sum is too low for 32 bits)
        const uint32_t keep = __ballot_sync(~0u, stays);
        const float last = -unordered(__reduce_max_sync(~0u, ordered(stays ? -value : -INFINITY)));
        const float next = unordered(__reduce_max_sync(~0u, ordered(open && !stays ? value : -INFINITY)));
        if (next > -INFINITY) sure = sure && last - next > unsure_groups(a.sigmoid, bias, inv, last, next);
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (e0 + j < E && !(keep >> ((e0 + j) / a.group_size * per) & 1u)) c[j] = -INFINITY;
        __syncwarp();
    }
    // order of the value, the last bits its place in the lane, lower places higher
    uint32_t key[EPL];
    constexpr uint32_t kPlace = EPL - 1;
#pragma unroll
    for (int j = 0; j < EPL; ++j) key[j] = (ordered(c[j]) & ~kPlace) | (kPlace - j);
    sort_words<EPL>(key);
    // One more than asked for, to see how near it came.  The lane that has the choice says so itself: where two have the same,
    // the lower one.
    chosen[warp][lane] = -1;
    __syncwarp();
    for (uint32_t r = 0; r <= a.top_k; ++r) {
        const uint32_t best = key[0] | kPlace, top = __reduce_max_sync(~0u, best);
        if (top <= (kClosed | kPlace)) break;
        const uint32_t same = __ballot_sync(~0u, best == top);
        const bool won = best == top && !(same & ((1u << lane) - 1));
        if (won && r < 32) chosen[warp][r] = (int)(e0 + kPlace - (key[0] & kPlace));
#pragma unroll
        for (int j = 0; j < EPL; ++j) key[j] = won ? (j + 1 < EPL ? key[j + 1] : 0u) : key[j];
    }
    __syncwarp();
    const int mine = chosen[warp][lane];  // lane r: choice r
    float xm = 0.f, sm = 0.f, bm = 0.f;
    if (mine >= 0) {
        xm = open_logit(ValueOf<DT>::get(row[mine]));
        sm = a.sigmoid ? sigmoid_of(xm) : expf(xm - m) * inv;
        bm = bias ? bias[mine] : 0.f;
    }
    const float y = scored ? sm + bm : xm;
    const float xn = __shfl_down_sync(~0u, xm, 1), bn = __shfl_down_sync(~0u, bm, 1), yn = __shfl_down_sync(~0u, y, 1);
    const float sn = __shfl_down_sync(~0u, sm, 1);
    const int other = __shfl_down_sync(~0u, mine, 1);
    // the larger score of the two; behind the last that is chosen there may be any (the largest of softmax is inv)
    const float top_score = !bias ? sm : lane + 1 == (int)a.top_k ? inv : fmaxf(sm, sn);
    // where 64 bits no longer tell scores of different logits apart
    if (mine >= 0 && !scored) sure = sure && (a.sigmoid ? xm < 16.f && xm > -600.f : xm - m > -600.f);
    // (two values that share a word's bits are out of order at most by what those bits are worth)
    if (lane < 31 && mine >= 0 && other >= 0 && !(xm == xn && bm == bn))
        sure = sure && y - yn > (scored ? unsure_values(a.sigmoid, top_score, y) : 1e-8f) + (DT == CIERA_FP32 || scored ? 1e-5f * fabsf(y) : 0.f);
    // The first that is not chosen is the same as the last that is: what shares their words' bits has not been seen.  Whatever is
    // near them without being the same is looked for in the whole row (closed groups too, for which 64 bits are no mistake).
    if ((DT == CIERA_FP32 || scored) && __any_sync(~0u, lane + 1 == (int)a.top_k && mine >= 0 && other >= 0 && xm == xn && bm == bn)) {
        const int from = (int)a.top_k - 1;
        const float xl = __shfl_sync(~0u, xm, from), bl = __shfl_sync(~0u, bm, from), yl = __shfl_sync(~0u, y, from), sl = __shfl_sync(~0u, top_score, from);
        const float margin = (scored ? unsure_values(a.sigmoid, sl, yl) : 1e-8f) + 1e-5f * fabsf(yl);
        for (uint32_t e = lane; e < E; e += 32) {
            const float xe = open_logit(ValueOf<DT>::get(row[e])), be = bias ? bias[e] : 0.f;
            const float ye = !scored ? xe : (a.sigmoid ? sigmoid_of(xe) : expf(xe - m) * inv) + be;
            if (xe > -INFINITY && ye > -INFINITY && !(xe == xl && be == bl)) sure = sure && fabsf(ye - yl) > margin;
        }
    }
    if (lane >= (int)a.top_k || mine < 0) sm = 0.f;
    const float sum = a.renormalise ? warp_sum(sm) : 1.f;
    if (mine >= 0 && sum < kSmallSum) sure = false;
    if (!__all_sync(~0u, sure)) {
        route_exact<DT, EPL>(row, a, bias, reinterpret_cast<unsigned long long*>(scratch), experts + t * a.top_k, weights + t * a.top_k);
        return;
    }
    if (a.renormalise) sm = sum > 0.f ? sm / sum : 0.f;
    if (lane < (int)a.top_k) {
        experts[t * a.top_k + lane] = mine;
        weights[t * a.top_k + lane] = sm * a.scale;
    }
}

// `lanes` lists of `KL` words in falling order, one in each of that many neighbouring lanes: all get the KL largest of all.
template <int KL, int L>
__device__ __forceinline__ void merge_lists(uint32_t (&list)[KL]) {
    constexpr int N = KL <= 16 ? 16 : KL <= 32 ? 32 : 64;
#pragma unroll
    for (int d = 1; d < L; d *= 2) {
        uint32_t t[N];
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = i < KL ? list[i] : 0u;
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            const uint32_t o = __shfl_xor_sync(~0u, list[i], d);
            t[N - 1 - i] = max(t[N - 1 - i], o);  // the N largest, falling and then rising
        }
#pragma unroll
        for (int step = N / 2; step; step /= 2)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(i & step)) {
                    const uint32_t hi = max(t[i], t[i + step]), lo = min(t[i], t[i + step]);
                    t[i] = hi;
                    t[i + step] = lo;
                }
#pragma unroll
        for (int i = 0; i < KL; ++i) list[i] = t[i];
    }
}

template <int KL>
__device__ __forceinline__ void put_in_list(uint32_t (&list)[KL], uint32_t v) {
#pragma unroll
    for (int i = KL - 1; i > 0; --i) list[i] = max(list[i], min(list[i - 1], v));
    list[0] = max(list[0], v);
}

template <int EPL>
constexpr int kTokenLanes = EPL <= 8 ? 4 : 16;  // L

// floats between the tokens' rows in shared memory: lanes that read 16 bytes together find them in banks of their own
__host__ __device__ inline uint32_t row_floats(uint32_t n_experts) { return (n_experts + 31) / 32 * 32 + 16; }
// of a warp: its tokens' rows and 32 group values a token
template <int EPL>
__host__ __device__ inline uint32_t warp_floats(uint32_t n_experts) {
    return 32 / kTokenLanes<EPL> * (row_floats(n_experts) + 32);
}

// KL: at least top_k + 2 (one more than asked for, to see how near it came, and one for values that share a word's bits)
template <int DT, int EPL, int KL>
__global__ void __launch_bounds__(kRouteWarps * 32, EPL <= 8 ? 4 : 2)
    route_kernel(const RouteArgs a, const value_t<DT>* __restrict__ logits, uint64_t n_tokens, uint64_t stride,
                 int whole, const float* __restrict__ bias, int32_t* __restrict__ experts, float* __restrict__ weights) {
    constexpr int L = kTokenLanes<EPL>, Q = (KL + L - 1) / L, V = 16 / sizeof(value_t<DT>);
    constexpr uint32_t tokens_each = 32 / L;
    extern __shared__ __align__(16) float route_smem[];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t E = a.n_experts, pitch = row_floats(E);
    float* rows = route_smem + warp * warp_floats<EPL>(E);
    float* group_values = rows + 32 / L * pitch;
    const bool grouped = a.top_groups < a.n_groups, scored = bias || grouped;
    const uint32_t place_mask = E > 1 ? ~0u >> __clz(E - 1) : 0u;  // a word's last bits: its place, lower places higher
    float* shifts = route_smem + kRouteWarps * warp_floats<EPL>(E);  // the bias, for the whole block
    for (uint32_t e = threadIdx.x; e < row_floats(E); e += kRouteWarps * 32) shifts[e] = bias && e < E ? (isnan(bias[e]) ? -INFINITY : bias[e]) : 0.f;
    __syncthreads();
    const uint64_t first = ((uint64_t)blockIdx.x * kRouteWarps + warp) * tokens_each;
    if (first >= n_tokens) return;
    const uint32_t here = (uint32_t)min((uint64_t)tokens_each, n_tokens - first);
    const uint32_t l = lane % L, mine = lane / L;
    const bool busy = mine < here;
    const uint64_t t = first + (busy ? mine : 0);
    float* row = rows + (busy ? mine : 0) * pitch;
    const value_t<DT>* row_logits = logits + t * stride;
    bool sure = true;
    uint32_t list[KL];
#pragma unroll
    for (int i = 0; i < KL; ++i) list[i] = 0;
    const auto put = [&](float y, uint32_t e) { put_in_list<KL>(list, (ordered(y) & ~place_mask) | ((place_mask - e) & place_mask)); };
    // Goes through the row, 16 bytes a lane at a time; f(values, the first one's place).  What is behind the row is closed.
    const auto each_piece = [&](auto&& f) {
#pragma unroll 2
        for (uint32_t e = l * V; e < E; e += L * V) {
            float x[V];
            if (whole && e + V <= E) {
                load_values<DT, V>(row_logits + e, x);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = e + j < E ? ValueOf<DT>::get(row_logits[e + j]) : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = open_logit(x[j]);
            f(x, e);
        }
    };
    float m = 0.f, inv = 1.f;
    if (!a.sigmoid) {
        m = -INFINITY;
        each_piece([&](const float(&x)[V], uint32_t) {
#pragma unroll
            for (int j = 0; j < V; ++j) m = fmaxf(m, x[j]);
        });
#pragma unroll
        for (int d = 1; d < L; d *= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
        if (m == -INFINITY) m = 0.f;  // nothing is open
        float sum = 0.f;
        each_piece([&](const float(&x)[V], uint32_t) {
#pragma unroll
            for (int j = 0; j < V; ++j) sum += expf(x[j] - m);
        });
#pragma unroll
        for (int d = 1; d < L; d *= 2) sum += __shfl_xor_sync(~0u, sum, d);
        inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
    }
    // what the choice goes by: the logits where there is no bias (scores rise with them), else s + b
    each_piece([&](const float(&x)[V], uint32_t e) {
        float y[V];
        if (scored) {
            const Pack<float, V> b = *reinterpret_cast<const Pack<float, V>*>(shifts + e);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float s = a.sigmoid ? __fdividef(1.f, 1.f + __expf(-x[j])) : expf(x[j] - m) * inv;
                y[j] = x[j] > -INFINITY ? s + b.v[j] : -INFINITY;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = x[j];
        }
        if (grouped) {
            if (busy) {
#pragma unroll
                for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(row + e + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) put(y[j], e + j);
        }
    });
    __syncwarp();
    if (grouped) {
        float* values = group_values + (busy ? mine : 0) * 32;
        const bool fours = !(a.group_size & 3);
        for (uint32_t g = l; g < a.n_groups; g += L) {
            float most = -INFINITY, second = -INFINITY;
            const auto see = [&](float y) {
                second = fmaxf(second, fminf(most, y));
                most = fmaxf(most, y);
            };
            if (fours) {
                const uint32_t n = a.group_size / 4;
                uint32_t e = l < n ? l : 0;  // (each lane begins elsewhere in its group: banks)
                for (uint32_t i = 0; i < n; ++i) {
                    const float4 y = *reinterpret_cast<const float4*>(row + g * a.group_size + 4 * e);
                    see(y.x);
                    see(y.y);
                    see(y.z);
                    see(y.w);
                    if (++e == n) e = 0;
                }
            } else {
                for (uint32_t i = 0; i < a.group_size; ++i) see(row[g * a.group_size + i]);
            }
            const float value = a.group_best > 1 && second > -INFINITY ? most + second : most;
            if (most > -INFINITY && value == -INFINITY) sure = false;  // (two open experts whose sum is too low for 32 bits)
            values[g] = value;
        }
        __syncwarp();
        // the groups that stay, and how far the first that goes is from the last of them
        uint32_t keep = 0;
        float last = INFINITY, next = -INFINITY;
        for (uint32_t g = l; g < a.n_groups; g += L) {
            const float v = values[g];
            uint32_t rank = 0;
            for (uint32_t i = 0; i < a.n_groups; ++i) {
                const float o = values[i];
                rank += o > v || (o == v && i < g);
            }
            if (v > -INFINITY && rank < a.top_groups) keep |= 1u << g, last = fminf(last, v);
            else next = fmaxf(next, v);
        }
#pragma unroll
        for (int d = 1; d < L; d *= 2) {
            last = fminf(last, __shfl_xor_sync(~0u, last, d));
            next = fmaxf(next, __shfl_xor_sync(~0u, next, d));
            keep |= __shfl_xor_sync(~0u, keep, d);
        }
        // (a bias of the other sign makes a sum small; the scores in it are still up to 1 each)
        if (next > -INFINITY) sure = sure && last - next > unsure_groups(a.sigmoid, bias, inv, last, next);
        for (uint32_t left = keep; left; left &= left - 1) {
            const uint32_t at = (__ffs(left) - 1) * a.group_size;
            if (fours) {
                for (uint32_t e = at + 4 * l; e < at + a.group_size; e += 4 * L) {
                    const float4 y = *reinterpret_cast<const float4*>(row + e);
                    put(y.x, e);
                    put(y.y, e + 1);
                    put(y.z, e + 2);
                    put(y.w, e + 3);
                }
            } else {
                for (uint32_t e = at + l; e < at + a.group_size; e += L) put(row[e], e);
            }
        }
        __syncwarp();
    }
    __syncwarp();
    merge_lists<KL, L>(list);

    // what is left, compared as it is: candidate i is with lane i % L
    uint32_t w[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) w[q] = 0;
#pragma unroll
    for (int i = 0; i < KL; ++i)
        if (l == i % L) w[i / L] = list[i];
    float x[Q], s[Q], y[Q], b[Q];
    uint32_t rank[Q];
    int at[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const bool open = w[q] > (kClosed | place_mask);
        at[q] = open ? (int)(place_mask - (w[q] & place_mask)) : -1;
        x[q] = open ? open_logit(ValueOf<DT>::get(row_logits[at[q]])) : -INFINITY;
        b[q] = open && bias ? bias[at[q]] : 0.f;
        s[q] = !open ? 0.f : a.sigmoid ? sigmoid_of(x[q]) : expf(x[q] - m) * inv;
        y[q] = !open ? -INFINITY : scored ? s[q] + b[q] : x[q];
        rank[q] = 0;
        // where 64 bits no longer tell scores of different logits apart
        if (open && !scored) sure = sure && (a.sigmoid ? x[q] < 16.f && x[q] > -600.f : x[q] - m > -600.f);
    }
    bool near[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) near[q] = false;
#pragma unroll
    for (int i = 0; i < KL; ++i) {
        const int from = lane / L * L + i % L;
        const float yi = __shfl_sync(~0u, y[i / L], from), xi = __shfl_sync(~0u, x[i / L], from), bi = __shfl_sync(~0u, b[i / L], from);
        const float si = bias ? __shfl_sync(~0u, s[i / L], from) : 0.f;  // (a bias may put a large score beside a small one)
        const int ei = __shfl_sync(~0u, at[i / L], from);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            rank[q] += yi > y[q] || (yi == y[q] && ei < at[q]);
            const float margin = scored ? unsure_values(a.sigmoid, fmaxf(s[q], si), y[q]) : 1e-8f;  // (logits below 16 this far apart: 64 bits tell)
            if (ei >= 0 && at[q] >= 0 && !(xi == x[q] && bi == b[q])) near[q] |= !(fabsf(yi - y[q]) > margin);
        }
    }
    // what is not on the list is at most what the last word of it may stand for (its score, where there is a bias, at most inv)
    const uint32_t last = list[KL - 1];
    const float beyond = last > (kClosed | place_mask) ? unordered(last | place_mask) : -INFINITY;
    const bool exact_words = DT != CIERA_FP32 && !scored && !(place_mask >> 13);  // (13 bits and more of such a logit are zero)
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (at[q] < 0 || rank[q] >= a.top_k) {
            if (q * L + (int)l < KL && at[q] >= 0 && rank[q] == a.top_k) sure = sure && !near[q];
            s[q] = 0.f;
            continue;
        }
        sure = sure && !near[q] && (exact_words || beyond == -INFINITY || y[q] - beyond > unsure_values(a.sigmoid, bias ? inv : s[q], y[q]));
        sum += s[q];
    }
    if (a.renormalise) {
#pragma unroll
        for (int d = 1; d < L; d *= 2) sum += __shfl_xor_sync(~0u, sum, d);
    }
    int found = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) found += at[q] >= 0;
#pragma unroll
    for (int d = 1; d < L; d *= 2) found += __shfl_xor_sync(~0u, found, d);
    if (a.renormalise && found && sum < kSmallSum) sure = false;
    if (busy) {
        int32_t* to = experts + t * a.top_k;
        float* tw = weights + t * a.top_k;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (at[q] < 0 || rank[q] >= a.top_k) continue;
            to[rank[q]] = at[q];
            tw[rank[q]] = (a.renormalise ? (sum > 0.f ? s[q] / sum : 0.f) : s[q]) * a.scale;
        }
        for (uint32_t r = found + l; r < a.top_k; r += L) to[r] = -1, tw[r] = 0.f;
    }
    uint32_t again = __ballot_sync(~0u, busy && !sure);
    while (again) {
        const uint32_t which = (__ffs(again) - 1) / L;
        again &= ~((L == 32 ? ~0u : (1u << L) - 1) << (which * L));
        __syncwarp();  // (the rows are its scratch; what was written above is written over)
        route_exact<DT, EPL>(logits + (first + which) * stride, a, bias, reinterpret_cast<unsigned long long*>(rows), experts + (first + which) * a.top_k,
                             weights + (first + which) * a.top_k);
    }
}

// dl = J_s^T ds: with p the chosen s over their sum, ds of choice j is scale * dw_j, or scale / sum * (dw_j - sum of p dw) when
// the weights are renormalised; softmax: dl = s * (ds - sum of ds s), where that sum is zero after renormalisation;
// sigmoid: dl = s * (1 - s) * ds.  A sum that 32 bits do not hold well: dl = p * (dw_j - sum of p dw) with p from 64 bits, since
// 1 / sum and s leave their range, and 1 - s is 1.
// LT lanes a token: half a warp for short rows (32768 tokens of 64 experts with a warp for each 8.9 us).
template <int LT, class T>
__device__ __forceinline__ T token_sum(T v) {
#pragma unroll
    for (int d = LT / 2; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}

// p * (d - sum of p d) over the token's choices, p the score of logit *at over their sum; for the whole warp
template <int DT, int LT>
__device__ __noinline__ float quotient_gradient(const value_t<DT>* at, bool some, int32_t sigmoid, float m, float d) {
    double p = 0.0;
    if (some) {
        const double x = open_logit(ValueOf<DT>::get(*at));
        p = exp(sigmoid ? -x : x - (double)m);
        if (sigmoid) p = 1.0 / (1.0 + p);
    }
    const double total = token_sum<LT>(p);
    p = total > 0.0 ? p / total : 0.0;
    return (float)(((double)d - token_sum<LT>((double)d * p)) * p);
}

template <int DT, int EPL, int LT>
__global__ void __launch_bounds__(kRouteWarps * 32)
    route_backward_kernel(const RouteArgs a, const value_t<DT>* __restrict__ logits, uint64_t n_tokens, uint64_t stride, int whole,
                          const int32_t* __restrict__ experts, const float* __restrict__ dweights,
                          value_t<DT>* __restrict__ dlogits, uint64_t dstride) {
    __shared__ __align__(16) float spread[kRouteWarps][32 * EPL];
    pdl_wait();
    const int full_lane = threadIdx.x & 31, warp = threadIdx.x >> 5, base = full_lane / LT * LT, lane = full_lane - base;
    const uint32_t E = a.n_experts, e0 = lane * EPL;
    float* all = spread[warp] + base * EPL;
    // a token's choice, its weights' gradients and its logits are on their way while the one before is done
    constexpr int kTokens = kRouteWarps * 32 / LT;  // of a block
    const uint64_t step = (uint64_t)gridDim.x * kTokens;
    uint64_t t = (uint64_t)blockIdx.x * kTokens + threadIdx.x / LT;
    float next_x[EPL], next_dw = 0.f;
    int next_id = -1;
    const auto fetch = [&](uint64_t of) {
        load_logits<DT, EPL>(logits + of * stride, E, whole, lane, next_x);
        if (lane < (int)a.top_k) next_id = experts[of * a.top_k + lane], next_dw = dweights[of * a.top_k + lane];
    };
    if (t < n_tokens) fetch(t);
    for (uint64_t first = (uint64_t)blockIdx.x * kTokens + warp * (32 / LT); first < n_tokens; first += step, t += step) {
        const bool here = t < n_tokens;  // (the warp's last token may have none beside it)
        const int id = here && (uint32_t)next_id < E ? next_id : -1;
        const float dw = id < 0 ? 0.f : next_dw;
        float x[EPL], s[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) x[j] = here ? open_logit(next_x[j]) : -INFINITY;
        if (t + step < n_tokens) fetch(t + step);
        float m = 0.f;
        if (a.sigmoid) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) s[j] = sigmoid_of(x[j]);
        } else {
            m = -INFINITY;
#pragma unroll
            for (int j = 0; j < EPL; ++j) m = fmaxf(m, x[j]);
            if constexpr (LT == 32) {
                m = unordered(__reduce_max_sync(~0u, ordered(m)));
            } else {
#pragma unroll
                for (int d = LT / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
            }
            if (m == -INFINITY) m = 0.f;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < EPL; ++j) sum += s[j] = expf(x[j] - m);
            sum = token_sum<LT>(sum);
            const float inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
#pragma unroll
            for (int j = 0; j < EPL; ++j) s[j] *= inv;
        }
        // the chosen scores
        Pack<float, EPL> put;
#pragma unroll
        for (int j = 0; j < EPL; ++j) put.v[j] = s[j];
        __syncwarp();
        *reinterpret_cast<Pack<float, EPL>*>(all + e0) = put;
        __syncwarp();
        const float sk = id < 0 ? 0.f : all[id];
        float d = dw * a.scale, dot = 0.f;
        if (a.renormalise) {
            const float total = token_sum<LT>(sk);
            const float it = total > 0.f ? __fdividef(1.f, total) : 0.f;
            const float of32 = (d - token_sum<LT>(d * sk) * it) * it;
            if (__any_sync(~0u, total < kSmallSum && id >= 0)) {
                const float of64 = quotient_gradient<DT, LT>(logits + (id >= 0 ? t * stride + id : 0), id >= 0, a.sigmoid, m, d);
                d = of32;
                if (total < kSmallSum) {  // (such that what follows leaves it as it is)
                    d = a.sigmoid ? 4.f * of64 : of64;
#pragma unroll
                    for (int j = 0; j < EPL; ++j) s[j] = a.sigmoid ? 0.5f : 1.f;
                }
            } else {
                d = of32;
            }
        } else if (!a.sigmoid) {
            dot = token_sum<LT>(d * sk);
        }
        // an expert that is named more than once gets the sum, in the order of the choices
        const uint32_t same = __match_any_sync(~0u, id < 0 ? -1 : id + base * 1024);
        if (__any_sync(~0u, id >= 0 && __popc(same) > 1)) {
            float sum = 0.f;
            for (uint32_t r = 0; r < a.top_k; ++r) {
                const float dr = __shfl_sync(~0u, d, base + (int)r);
                if (same >> (base + r) & 1u) sum += dr;
            }
            d = sum;
        }
#pragma unroll
        for (int j = 0; j < EPL; ++j) put.v[j] = 0.f;
        __syncwarp();
        *reinterpret_cast<Pack<float, EPL>*>(all + e0) = put;
        __syncwarp();
        if (id >= 0) all[id] = d;  // (the same sum from each of the same)
        __syncwarp();
        float ds[EPL];
        const Pack<float, EPL> mine = *reinterpret_cast<const Pack<float, EPL>*>(all + e0);
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            ds[j] = a.sigmoid ? mine.v[j] * s[j] * (1.f - s[j]) : s[j] * (mine.v[j] - dot);
            if (x[j] == -INFINITY) ds[j] = 0.f;
        }
        if (!here) continue;
        value_t<DT>* to = dlogits + t * dstride + e0;
        if (whole && e0 + EPL <= E) {
            store_values<DT, EPL>(to, ds);
        } else {
#pragma unroll
            for (int j = 0; j < EPL; ++j)
                if (e0 + j < E) to[j] = ValueOf<DT>::put(ds[j]);
        }
    }
}

static int route_args(const ciera_route_config* c, RouteArgs* a) {
    if (!c) return CIERA_ERR_INVALID_ARG;
    if (c->n_experts < 1 || c->n_experts > 1024 || c->n_groups < 1 || c->n_groups > 32 || c->n_experts % c->n_groups ||
        c->top_groups < 1 || c->top_groups > c->n_groups || c->group_best < 1 || c->group_best > 2 || c->top_k < 1 ||
        c->top_k > 32 || c->top_k > c->top_groups * (c->n_experts / c->n_groups) ||
        (c->score != CIERA_SCORE_SOFTMAX && c->score != CIERA_SCORE_SIGMOID) ||
        (c->renormalise != 0 && c->renormalise != 1) || !isfinite(c->scale))
        return CIERA_ERR_INVALID_ARG;
    *a = RouteArgs{c->n_experts, c->top_k, c->n_groups, c->top_groups, c->group_best, c->n_experts / c->n_groups,
                   c->score == CIERA_SCORE_SIGMOID, c->renormalise, c->scale};
    return CIERA_OK;
}

// f(values per lane as a constant) for a row of n experts
template <class F>
static void with_row(uint32_t n, F&& f) {
    if (n <= 64) f(std::integral_constant<int, 2>());
    else if (n <= 256) f(std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 32>());
}
// f(length of the lists as a constant)
template <class F>
static void with_list(uint32_t top_k, F&& f) {
    if (top_k <= 8) f(std::integral_constant<int, 10>());
    else if (top_k <= 16) f(std::integral_constant<int, 18>());
    else f(std::integral_constant<int, 34>());
}

// whether rows may be read EPL values at a time, in pieces of at most 16 bytes
static bool whole_rows(const void* p, uint64_t stride, uint64_t value_bytes, uint64_t epl) {
    const uint64_t piece = epl * value_bytes < 16 ? epl * value_bytes : 16;
    return !(((uint64_t)p | stride * value_bytes) & (piece - 1));
}

static uint32_t route_grid(uint64_t n_tokens) {
    const uint64_t blocks = (n_tokens + kRouteWarps - 1) / kRouteWarps;
    return (uint32_t)(blocks < 148 * 16 ? blocks : 148 * 16);
}

}  // namespace ciera

using namespace ciera;

extern "C" int ciera_route(const ciera_route_config* config, int dtype, const void* logits_dev, uint64_t n_tokens,
                           uint64_t logits_stride, const float* bias_dev, int32_t* experts_dev, float* weights_dev,
                           void* stream) {
    RouteArgs a;
    const int rc = route_args(config, &a);
    if (rc) return rc;
    if (n_tokens > kMaxExtent || (n_tokens > 1 && logits_stride < a.n_experts)) return CIERA_ERR_INVALID_ARG;
    if (n_tokens && (!logits_dev || !experts_dev || !weights_dev)) return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(logits_dev, dtype_bytes(dtype)) || !aligned_to(bias_dev, 4) || !aligned_to(experts_dev, 4) ||
        !aligned_to(weights_dev, 4))
        return CIERA_ERR_MISALIGNED;
    cudaError_t e = cudaSuccess;
    const bool known = with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (!n_tokens) return;
        with_row(a.n_experts, [&](auto epl) {
            // A warp for each token while all of them have room on the GPU, else 32 / L tokens a warp (one token 2.5 us against
            // 5.8, 16384 tokens of 256 experts in 8 groups 43 us against 24; spread over more warps, 6000 of 256 22.8 us against 18.2).
            if (n_tokens < 148 * 32) {
                constexpr int EPL = decltype(epl)::value;
                e = launch_after(route_few_kernel<DT, EPL>, dim3((uint32_t)((n_tokens + kRouteWarps - 1) / kRouteWarps)), kRouteWarps * 32,
                                 sizeof(float) * kRouteWarps * 2 * a.n_experts /* at most 32 KB */, (cudaStream_t)stream, a, (const value_t<DT>*)logits_dev,
                                 n_tokens, logits_stride, whole_rows(logits_dev, logits_stride, dtype_bytes(DT), EPL), bias_dev, experts_dev,
                                 weights_dev);
                return;
            }
            with_list(a.top_k, [&](auto kl) {
                constexpr int EPL = decltype(epl)::value, KL = decltype(kl)::value;
                const int whole = whole_rows(logits_dev, logits_stride, dtype_bytes(DT), 16 / dtype_bytes(DT));
                // (also what a token that is done again takes) at most 42 KB
                const size_t smem = sizeof(float) * (kRouteWarps * warp_floats<EPL>(a.n_experts) + row_floats(a.n_experts));
                constexpr uint32_t tokens_each = 32 / kTokenLanes<EPL>;  // of a warp
                const uint64_t blocks = (n_tokens + (uint64_t)tokens_each * kRouteWarps - 1) / ((uint64_t)tokens_each * kRouteWarps);
                e = launch_after(route_kernel<DT, EPL, KL>, dim3((uint32_t)blocks), kRouteWarps * 32, smem, (cudaStream_t)stream, a,
                                 (const value_t<DT>*)logits_dev, n_tokens, logits_stride, whole, bias_dev, experts_dev,
                                 weights_dev);
            });
        });
    });
    if (!known) return CIERA_ERR_INVALID_ARG;
    if (e != cudaSuccess) return record_cuda_error(e);
    if (n_tokens) count_launch();
    return CIERA_OK;
}

extern "C" int ciera_route_backward(const ciera_route_config* config, int dtype, const void* logits_dev, uint64_t n_tokens,
                                    uint64_t logits_stride, const int32_t* experts_dev, const float* dweights_dev,
                                    void* dlogits_dev, uint64_t dlogits_stride, void* stream) {
    RouteArgs a;
    const int rc = route_args(config, &a);
    if (rc) return rc;
    if (n_tokens > kMaxExtent || (n_tokens > 1 && (logits_stride < a.n_experts || dlogits_stride < a.n_experts)))
        return CIERA_ERR_INVALID_ARG;
    if (n_tokens && (!logits_dev || !experts_dev || !dweights_dev || !dlogits_dev)) return CIERA_ERR_INVALID_ARG;
    if (!aligned_to(logits_dev, dtype_bytes(dtype)) || !aligned_to(dlogits_dev, dtype_bytes(dtype)) ||
        !aligned_to(experts_dev, 4) || !aligned_to(dweights_dev, 4))
        return CIERA_ERR_MISALIGNED;
    cudaError_t e = cudaSuccess;
    const bool known = with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (!n_tokens) return;
        with_row(a.n_experts, [&](auto epl) {
            const auto go = [&](auto each, auto lanes) {
                constexpr int EPL = decltype(each)::value, LT = decltype(lanes)::value;
                const int whole = whole_rows(logits_dev, logits_stride, dtype_bytes(DT), EPL) &&
                                  whole_rows(dlogits_dev, dlogits_stride, dtype_bytes(DT), EPL);
                e = launch_after(route_backward_kernel<DT, EPL, LT>, dim3(route_grid((n_tokens + 32 / LT - 1) / (32 / LT))), kRouteWarps * 32, 0,
                                 (cudaStream_t)stream, a, (const value_t<DT>*)logits_dev, n_tokens, logits_stride, whole, experts_dev,
                                 dweights_dev, (value_t<DT>*)dlogits_dev, dlogits_stride);
            };
            constexpr int EPL = decltype(epl)::value;
            if constexpr (EPL == 2) {
                if (a.top_k <= 16) {
                    go(std::integral_constant<int, 4>(), std::integral_constant<int, 16>());
                    return;
                }
            }
            go(epl, std::integral_constant<int, 32>());
        });
    });
    if (!known) return CIERA_ERR_INVALID_ARG;
    if (e != cudaSuccess) return record_cuda_error(e);
    if (n_tokens) count_launch();
    return CIERA_OK;
}
