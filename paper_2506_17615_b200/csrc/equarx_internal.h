// What the library's two host files share.
#pragma once
#include <cuda_runtime.h>

namespace equarx {
// cudaSuccess, or what EQUARX_INJECT_LAUNCH_ERROR asks every launch to report
cudaError_t launch_error_to_inject();
// false with EQUARX_PDL=0
bool dependent_launches();
// records `e` for equarx_last_cuda_error() and returns EQUARX_ERR_CUDA
int cuda_failure(cudaError_t e);
}  // namespace equarx
