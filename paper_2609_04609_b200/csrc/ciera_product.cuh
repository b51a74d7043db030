// What the products of 8-bit and of 4-bit operands share: writing out finished sums, tensor maps of operands.
#pragma once

#include <cuda.h>

#include "ciera_numeric.cuh"
#include "ciera_tensor.cuh"

namespace ciera {

// Two sums rounded to a 16-bit type, the first in the low half.
template <int DT>
__device__ __forceinline__ uint32_t pack_two(uint32_t lo, uint32_t hi) {
    const float x = __uint_as_float(lo), y = __uint_as_float(hi);
    if constexpr (DT == CIERA_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}

// Writes 32 columns x 32 rows of out of which the lane has column `col` in r: neighbouring columns are in neighbouring lanes, so
// a row goes out as it is, 16-bit values two at a time: an even lane puts row c's together, its neighbour row c + 1's.
template <int DT>
__device__ __forceinline__ void write_part(const uint32_t (&r)[32], value_t<DT>* out, uint64_t stride, uint32_t row, uint32_t rows,
                                           uint32_t col, uint32_t cols, bool wide, int lane) {
    if constexpr (DT == CIERA_FP32) {
        uint32_t* to = reinterpret_cast<uint32_t*>(out + row * stride + col);
        if (col >= cols) return;
        if (row + 32 <= rows) {
#pragma unroll
            for (int c = 0; c < 32; ++c, to += stride) *to = r[c];
        } else {
#pragma unroll
            for (int c = 0; c < 32; ++c, to += stride)
                if (row + c < rows) *to = r[c];
        }
    } else if (wide) {
        const uint32_t odd = lane & 1;
        uint32_t* to = reinterpret_cast<uint32_t*>(out + (row + odd) * stride + (col - odd));
        const bool some = col - odd < cols;  // (cols is even)
        const bool all = row + 32 <= rows;
#pragma unroll
        for (int c = 0; c < 32; c += 2, to += stride) {
            const uint32_t other = __shfl_xor_sync(~0u, odd ? r[c] : r[c + 1], 1);
            const uint32_t both = odd ? pack_two<DT>(other, r[c + 1]) : pack_two<DT>(r[c], other);
            if (some && (all || row + c + odd < rows)) *to = both;
        }
    } else {
        value_t<DT>* to = out + row * stride + col;
#pragma unroll
        for (int c = 0; c < 32; ++c, to += stride)
            if (col < cols && row + c < rows) *to = ValueOf<DT>::put(__uint_as_float(r[c]));
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return f;
}

// Tiles of 128 bytes x `box` rows of [matrices][rows, k] bytes; what lies outside arrives as zero.
inline bool operand_map(CUtensorMap* map, const void* p, uint64_t k, uint64_t rows, uint64_t matrices, uint64_t stride,
                        uint64_t matrix_stride, uint32_t box) {
    const uint64_t line = (k + 15) & ~15ull;
    if (rows <= 1) stride = line;  // (never stepped by)
    if (matrices <= 1) matrix_stride = stride;
    const cuuint64_t dims[3] = {k, rows, matrices}, strides[2] = {stride, matrix_stride};
    const cuuint32_t boxes[3] = {128, box, 1}, steps[3] = {1, 1, 1};
    return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(p), dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the current device and its SMs
inline int device_and_sms(int* dev, int* n) {
    static std::atomic<int> known[64];
    cudaError_t e = cudaGetDevice(dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (*dev < 64 && (*n = known[*dev].load(std::memory_order_relaxed)) > 0) return CIERA_OK;
    e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, *dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (*dev < 64) known[*dev].store(*n, std::memory_order_relaxed);
    return CIERA_OK;
}

}  // namespace ciera
