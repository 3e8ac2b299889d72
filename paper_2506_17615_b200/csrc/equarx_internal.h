// What the library's host files share.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace equarx {
// cudaSuccess, or what EQUARX_INJECT_LAUNCH_ERROR asks every launch to report
cudaError_t launch_error_to_inject();
// false with EQUARX_PDL=0
bool dependent_launches();
// records `e` for equarx_last_cuda_error() and returns EQUARX_ERR_CUDA
int cuda_failure(cudaError_t e);
// clusters of 1 .. 8 CTAs that run at one time on the current device when each CTA has an SM to itself
int resident_clusters(int (&out)[9]);
// for tests: launches a wait of so many polls that runs out, counted with those of the adapters' kernels
cudaError_t adapters_give_up(uint32_t polls);
// waits of the adapters' kernels that gave up on the current device since the last call
cudaError_t adapters_gave_up(uint32_t& seen);
}  // namespace equarx
