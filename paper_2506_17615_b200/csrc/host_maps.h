// Tensor maps of the host files whose kernels use TMA.
#pragma once
#include <cuda.h>

#include "host_common.h"

namespace equarx {
namespace host {

constexpr int kMapBytes = 128;            // of a box's rows, with the 128-byte swizzle or none

// The driver's encoder is looked up through the runtime, so the library needs no link to the driver.
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline Encode encoder() {
    static Encode fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<Encode>(p);
    }();
    return fn;
}

// rows x inner elements of 1 or 2 bytes, row stride in bytes; boxes of box_rows x 128 bytes (64 with the
// 64-byte swizzle); elements outside the matrix read as zero
inline int make_map(CUtensorMap& map, const void* base, size_t elem, size_t inner, size_t rows, size_t stride, size_t box_rows,
             CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {stride};
    const cuuint32_t box[2] = {cuuint32_t((swizzle == CU_TENSOR_MAP_SWIZZLE_64B ? 64 : kMapBytes) / elem), cuuint32_t(box_rows)},
                     steps[2] = {1, 1};
    const Encode fn = encoder();
    if (!fn) return cuda_failure(cudaErrorNotSupported);
    const CUresult r = fn(&map, elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2,
                          const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? EQUARX_OK : cuda_failure(cudaErrorInvalidValue);
}

}  // namespace host
}  // namespace equarx
