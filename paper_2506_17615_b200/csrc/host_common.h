// What the host files of the calls for one GPU share: checks of arguments, facts about the device, launches.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <mutex>

#include "../../include/equarx.h"
#include "equarx_internal.h"

namespace equarx {
namespace host {

constexpr size_t kMaxDim = size_t(1) << 30;
constexpr size_t kBigSmem = 227 * 1024;

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }
inline size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------- checks
struct Span {
    const void* p;
    size_t bytes;           // from the first to the last
    size_t width, stride;   // of a row, in bytes; a buffer is one row
    Span(const void* p, size_t bytes) : Span(p, bytes, bytes, 0) {}
    Span(const void* p, size_t bytes, size_t width, size_t stride) : p(p), bytes(bytes), width(width), stride(stride) {}
};
inline Span matrix(const void* p, size_t rows, size_t cols, size_t ld, size_t size) {
    return rows > 1 ? Span(p, ((rows - 1) * ld + cols) * size, cols * size, ld * size) : Span(p, rows * cols * size);
}
// Matrices of one row stride may share its rows, each with columns of its own (the two halves of a wider buffer):
// one's rows then begin after the other's, counted from there, and end before the other's next ones.  Matrices of
// different strides are kept apart as a whole.
inline bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    if (!(a.bytes && b.bytes && a.p && b.p && x < y + b.bytes && y < x + a.bytes)) return false;
    const size_t stride = std::max(a.stride, b.stride);
    if (!stride || (a.stride && b.stride && a.stride != b.stride)) return true;
    const size_t after = y >= x ? (y - x) % stride : (stride - (x - y) % stride) % stride;
    return after < a.width || after + b.width > stride;
}
// no output may meet an input or another output
inline int check_overlap(std::initializer_list<Span> in, std::initializer_list<Span> out) {
    for (auto o = out.begin(); o != out.end(); ++o) {
        for (const Span& i : in)
            if (overlap(*o, i)) return EQUARX_ERR_ALIAS;
        for (auto q = out.begin(); q != o; ++q)
            if (overlap(*o, *q)) return EQUARX_ERR_ALIAS;
    }
    return EQUARX_OK;
}
inline bool bad_dim(size_t d) { return d == 0 || d > kMaxDim; }
inline bool bad_ld(size_t ld, size_t cols) { return ld < cols || ld > kMaxDim; }
inline bool is_16bit(int dtype) { return dtype == EQUARX_BF16 || dtype == EQUARX_FP16; }
inline bool is_float(int dtype) { return is_16bit(dtype) || dtype == EQUARX_FP32; }
inline bool is_act(int a) { return a == EQUARX_ACT_SILU || a == EQUARX_ACT_GELU_TANH; }
// bytes, at most 32, that a base and a row stride are multiples of
inline int unit_of(const void* p, size_t ld, size_t size) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (ld * size) | 32;
    return int(bits & (~bits + 1));
}
inline size_t size_of(int dtype) { return dtype == EQUARX_FP32 ? 4 : 2; }

// ---------------------------------------------------------------- device facts, constant for the process
// (kept in arrays of a fixed size: nothing here may throw into a C caller)
constexpr int kMaxDevices = 64, kMaxKernels = 128;

struct DeviceFacts {
    int sms = 0;                 // 0: not looked up yet
    int clusters[9] = {};        // clusters of so many CTAs that run at one time
    bool has_clusters = false;
};
inline std::mutex g_facts_mutex;
inline DeviceFacts g_facts[kMaxDevices];

inline int device_index(int& dev) {
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_failure(e);
    return dev < kMaxDevices ? EQUARX_OK : cuda_failure(cudaErrorInvalidDevice);
}

inline int current_device(int& sms) {
    int dev;
    if (const int st = device_index(dev)) return st;
    std::lock_guard<std::mutex> lock(g_facts_mutex);
    if (!g_facts[dev].sms) {
        const cudaError_t e = cudaDeviceGetAttribute(&g_facts[dev].sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return cuda_failure(e);
    }
    sms = g_facts[dev].sms;
    return EQUARX_OK;
}

// ---------------------------------------------------------------- launches
// kernels that need more than 48 KB of shared memory ask for it once per device
// (`all`: of the SM's L1, as much as can be is shared memory, for kernels that want several CTAs on an SM)
inline cudaError_t allow_smem(const void* kernel, bool all) {
    struct Entry {
        const void* kernel;
        uint64_t devices;
    };
    static std::mutex mu;
    static Entry seen[kMaxKernels];
    static int count = 0;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    int i = 0;
    while (i < count && seen[i].kernel != kernel) ++i;
    const uint64_t bit = dev < kMaxDevices ? uint64_t(1) << dev : 0;
    if (i < count && (seen[i].devices & bit)) return cudaSuccess;
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, kernel);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kBigSmem - fa.sharedSizeBytes));
    if (e == cudaSuccess && all)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess && i < kMaxKernels) {
        seen[i].kernel = kernel;
        seen[i].devices |= bit;
        count = std::max(count, i + 1);
    }
    return e;
}

template <typename Args>
int launch(void (*kernel)(Args), dim3 grid, int threads, size_t smem, unsigned cluster, const Args& args,
           cudaStream_t stream, bool all_shared = false) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
    if (dependent_launches()) {      // every kernel waits for the stream's earlier work before it reads
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    cudaError_t e = launch_error_to_inject();
    // (48 KB hold what a kernel declares, too)
    if (e == cudaSuccess && (smem > 32 * 1024 || all_shared)) e = allow_smem(reinterpret_cast<const void*>(kernel), all_shared);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kernel, args);
    return e == cudaSuccess ? EQUARX_OK : cuda_failure(e);
}

#define TRY(call)                              \
    do {                                       \
        if (const int try_status = (call)) return try_status; \
    } while (0)

}  // namespace host
}  // namespace equarx
