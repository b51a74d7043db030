// Routing of tokens to experts, and its gradient.  A warp per token; expert e of a row is value e / 32 of lane e % 32.
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

// a logit as it counts: closed (-inf) or finite
__device__ __forceinline__ float open_logit(float x) { return isnan(x) ? -INFINITY : fminf(x, 3.402823466e38f); }

// One token's choice in 64 bits.  x: the lane's logits (-inf: closed).  c: E doubles of the warp's own in shared memory.
template <int EPL>
__device__ void route_exact(const float (&x)[EPL], const RouteArgs& a, const float* __restrict__ bias, double* c, int lane,
                            int32_t* __restrict__ experts, float* __restrict__ weights) {
    const int E = (int)a.n_experts;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < EPL; ++j) m = fmaxf(m, x[j]);
    m = warp_max(m);
    double s[EPL], v[EPL];
    double total = 0.0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        if (x[j] == -INFINITY) s[j] = 0.0;
        else if (a.sigmoid) s[j] = 1.0 / (1.0 + exp(-(double)x[j]));
        else total += s[j] = exp((double)x[j] - (double)m);
    }
    if (!a.sigmoid) {
        total = warp_sum(total);
#pragma unroll
        for (int j = 0; j < EPL; ++j) s[j] = total > 0.0 ? s[j] / total : 0.0;
    }
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        const int e = j * 32 + lane;
        v[j] = s[j] + (bias && e < E ? (double)bias[e] : 0.0);
        if (x[j] == -INFINITY || isnan(v[j])) v[j] = -INFINITY;
    }
    if (a.top_groups < a.n_groups) {
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (j * 32 + lane < E) c[j * 32 + lane] = v[j];
        __syncwarp();
        double g = -INFINITY;  // lane i: value of group i
        if (lane < (int)a.n_groups) {
            double first = -INFINITY, second = -INFINITY;
            for (uint32_t i = 0; i < a.group_size; ++i) {
                const double y = c[lane * a.group_size + i];
                if (y > first) second = first, first = y;
                else if (y > second) second = y;
            }
            g = first;
            if (a.group_best > 1 && second > -INFINITY) g += second;
        }
        __syncwarp();
        uint32_t keep = 0;
        bool mine = g > -INFINITY;
        for (uint32_t r = 0; r < a.top_groups; ++r) {
            double best = mine ? g : -INFINITY;
#pragma unroll
            for (int d = 16; d; d >>= 1) best = fmax(best, __shfl_xor_sync(~0u, best, d));
            const uint32_t at = __ballot_sync(~0u, mine && g == best);
            if (!at) break;
            const int w = __ffs(at) - 1;
            keep |= 1u << w;
            if (lane == w) mine = false;
        }
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const uint32_t e = j * 32 + lane;
            if (e < a.n_experts && !((keep >> (e / a.group_size)) & 1u)) v[j] = -INFINITY;
        }
    }
    // lane i ends up with choice i
    int chosen = -1;
    double ws = 0.0, sum = 0.0;
    for (uint32_t r = 0; r < a.top_k; ++r) {
        double best = -INFINITY, bs = 0.0;
        int be = 1 << 30;
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (v[j] > best) best = v[j], be = j * 32 + lane, bs = s[j];
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const double ob = __shfl_xor_sync(~0u, best, d), os = __shfl_xor_sync(~0u, bs, d);
            const int oe = __shfl_xor_sync(~0u, be, d);
            if (ob > best || (ob == best && oe < be)) best = ob, be = oe, bs = os;
        }
        if (be == 1 << 30) break;
        if (lane == (int)r) chosen = be, ws = bs;
        sum += bs;
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (j * 32 + lane == be) v[j] = -INFINITY;
    }
    if (lane < (int)a.top_k) {
        if (a.renormalise) ws = sum > 0.0 ? ws / sum : 0.0;
        experts[lane] = chosen;
        weights[lane] = (float)(ws * (double)a.scale);
    }
}

template <int DT, int EPL>
__global__ void __launch_bounds__(kRouteWarps * 32) route_kernel(const RouteArgs a, const value_t<DT>* __restrict__ logits,
                                                                uint64_t n_tokens, uint64_t stride,
                                                                const float* __restrict__ bias, int32_t* __restrict__ experts,
                                                                float* __restrict__ weights) {
    extern __shared__ double route_smem[];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double* c = route_smem + (size_t)warp * a.n_experts;
    for (uint64_t t = (uint64_t)blockIdx.x * kRouteWarps + warp; t < n_tokens; t += (uint64_t)gridDim.x * kRouteWarps) {
        float x[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const uint32_t e = j * 32 + lane;
            x[j] = e < a.n_experts ? open_logit(ValueOf<DT>::get(logits[t * stride + e])) : -INFINITY;
        }
        route_exact<EPL>(x, a, bias, c, lane, experts + t * a.top_k, weights + t * a.top_k);
    }
}

// dl = J_s^T ds: with p the chosen s over their sum, ds of choice j is scale * dw_j, or scale / sum * (dw_j - sum of p dw) when
// the weights are renormalised; softmax: dl = s * (ds - sum of ds s), where that sum is zero after renormalisation;
// sigmoid: dl = s * (1 - s) * ds.
template <int DT, int EPL>
__global__ void __launch_bounds__(kRouteWarps * 32)
    route_backward_kernel(const RouteArgs a, const value_t<DT>* __restrict__ logits, uint64_t n_tokens, uint64_t stride,
                          const int32_t* __restrict__ experts, const float* __restrict__ dweights,
                          value_t<DT>* __restrict__ dlogits, uint64_t dstride) {
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint64_t t = (uint64_t)blockIdx.x * kRouteWarps + warp; t < n_tokens; t += (uint64_t)gridDim.x * kRouteWarps) {
        const value_t<DT>* row = logits + t * stride;
        float x[EPL], s[EPL];
        int id = -1;
        float dw = 0.f, xk = -INFINITY;
        if (lane < (int)a.top_k) {
            id = experts[t * a.top_k + lane];
            if ((uint32_t)id >= a.n_experts) id = -1;
            if (id >= 0) {
                dw = dweights[t * a.top_k + lane];
                xk = open_logit(ValueOf<DT>::get(row[id]));
            }
        }
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const uint32_t e = j * 32 + lane;
            x[j] = e < a.n_experts ? open_logit(ValueOf<DT>::get(row[e])) : -INFINITY;
            m = fmaxf(m, x[j]);
        }
        float inv = 1.f, sk;
        if (a.sigmoid) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) s[j] = 1.f / (1.f + expf(-x[j]));
            sk = 1.f / (1.f + expf(-xk));
        } else {
            m = warp_max(m);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < EPL; ++j) sum += s[j] = x[j] == -INFINITY ? 0.f : expf(x[j] - m);
            sum = warp_sum(sum);
            inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
            for (int j = 0; j < EPL; ++j) s[j] *= inv;
            sk = xk == -INFINITY ? 0.f : expf(xk - m) * inv;
        }
        float d = dw * a.scale, dot = 0.f;
        if (a.renormalise) {
            const float total = warp_sum(sk);
            const float it = total > 0.f ? 1.f / total : 0.f;
            d = (d - warp_sum(d * sk) * it) * it;
        } else if (!a.sigmoid) {
            dot = warp_sum(d * sk);
        }
        float ds[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) ds[j] = 0.f;
        for (uint32_t r = 0; r < a.top_k; ++r) {
            const int e = __shfl_sync(~0u, id, (int)r);
            const float dr = __shfl_sync(~0u, d, (int)r);
#pragma unroll
            for (int j = 0; j < EPL; ++j)
                if (e == j * 32 + lane) ds[j] += dr;
        }
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const uint32_t e = j * 32 + lane;
            if (e >= a.n_experts) continue;
            float g = a.sigmoid ? ds[j] * s[j] * (1.f - s[j]) : s[j] * (ds[j] - dot);
            if (x[j] == -INFINITY) g = 0.f;
            dlogits[t * dstride + e] = ValueOf<DT>::put(g);
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
    if (n <= 32) f(std::integral_constant<int, 1>());
    else if (n <= 64) f(std::integral_constant<int, 2>());
    else if (n <= 128) f(std::integral_constant<int, 4>());
    else if (n <= 256) f(std::integral_constant<int, 8>());
    else if (n <= 512) f(std::integral_constant<int, 16>());
    else f(std::integral_constant<int, 32>());
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
            const size_t smem = a.top_groups < a.n_groups ? sizeof(double) * kRouteWarps * a.n_experts : 0;  // at most 32 KB
            e = launch_after(route_kernel<DT, decltype(epl)::value>, dim3(route_grid(n_tokens)), kRouteWarps * 32, smem,
                             (cudaStream_t)stream, a, (const value_t<DT>*)logits_dev, n_tokens, logits_stride, bias_dev,
                             experts_dev, weights_dev);
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
            e = launch_after(route_backward_kernel<DT, decltype(epl)::value>, dim3(route_grid(n_tokens)), kRouteWarps * 32, 0,
                             (cudaStream_t)stream, a, (const value_t<DT>*)logits_dev, n_tokens, logits_stride, experts_dev,
                             dweights_dev, (value_t<DT>*)dlogits_dev, dlogits_stride);
        });
    });
    if (!known) return CIERA_ERR_INVALID_ARG;
    if (e != cudaSuccess) return record_cuda_error(e);
    if (n_tokens) count_launch();
    return CIERA_OK;
}
