// Values of the three precisions as fp32, one at a time or in aligned groups, and scale bytes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "ciera_internal.cuh"

namespace ciera {

template <int DT>
struct ValueOf;
template <>
struct ValueOf<CIERA_BF16> {
    using type = __nv_bfloat16;
    static __device__ __forceinline__ float get(type v) { return __bfloat162float(v); }
    static __device__ __forceinline__ type put(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct ValueOf<CIERA_FP32> {
    using type = float;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct ValueOf<CIERA_FP16> {
    using type = __half;
    static __device__ __forceinline__ float get(type v) { return __half2float(v); }
    static __device__ __forceinline__ type put(float v) { return __float2half_rn(v); }
};
template <int DT>
using value_t = typename ValueOf<DT>::type;

// N neighbouring values in one access; the address is a multiple of N values (and of at most 16 bytes).
template <class T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack {
    T v[N];
};
template <int DT, int N>
__device__ __forceinline__ void load_values(const value_t<DT>* p, float (&out)[N]) {
    const Pack<value_t<DT>, N> r = *reinterpret_cast<const Pack<value_t<DT>, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = ValueOf<DT>::get(r.v[i]);
}
template <int DT, int N>
__device__ __forceinline__ void store_values(value_t<DT>* p, const float (&in)[N]) {
    Pack<value_t<DT>, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = ValueOf<DT>::put(in[i]);
    *reinterpret_cast<Pack<value_t<DT>, N>*>(p) = r;
}

// Calls f with the precision as a constant; false for a code that is none.
template <class F>
bool with_dtype(int dtype, F&& f) {
    switch (dtype) {
        case CIERA_BF16: f(std::integral_constant<int, CIERA_BF16>()); return true;
        case CIERA_FP32: f(std::integral_constant<int, CIERA_FP32>()); return true;
        case CIERA_FP16: f(std::integral_constant<int, CIERA_FP16>()); return true;
        default: return false;
    }
}
inline uint64_t dtype_bytes(int dtype) { return dtype == CIERA_FP32 ? 4 : 2; }
inline bool aligned_to(const void* p, uint64_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

constexpr int kFp8Block = CIERA_FP8_BLOCK;
constexpr uint64_t kMaxExtent = (1ull << 31) - 256;

}  // namespace ciera
