// C ABI of the residual addition with RMS norm (include/equarx.h): argument checks, launches.
#include <cmath>

#include "host_common.h"
#include "norm_kernels.cuh"

namespace {

using namespace equarx;
using namespace equarx::ff;
using namespace equarx::host;

inline bool is_weight(int dtype, int type) { return type == dtype || type == EQUARX_FP32; }
inline bool bad_value(double eps, double offset) { return !(eps >= 0.0) || std::isinf(eps) || !std::isfinite(offset); }

// elements of an access: rows that start on multiples of 16, 4 or 2 bytes
struct Access {
    int unit = 32;
    void add(const void* p, size_t ld) {
        if (p) unit = std::min(unit, unit_of(p, ld, 2));
    }
    // fp32 is read in words of 16 bytes or of 4
    void add_weight(const void* p, bool fp32) {
        if (!fp32) add(p, 0);
        else if (!aligned(p, 16)) unit = std::min(unit, 4);
    }
    int width() const { return unit >= 16 ? 8 : unit >= 4 ? 2 : 1; }
};

// Groups of 8 columns for each thread of the backward pass: as few threads as hold a row, up to 224 of them, since each
// thread's part in the row's reduction costs as much as 8 columns do.  0: a row that no CTA holds.
inline int grad_groups(size_t cols) { return cols > size_t(kGradGroups * kGradColumns) ? 0 : int(ceil_div(cols, kGradColumns)); }
inline int grad_threads(size_t cols) {
    const int groups = grad_groups(cols);
    return groups ? int(up(ceil_div(cols, 8 * groups), 32)) : kGradThreads;
}

// Rows up to which the CTAs of the backward pass are one cluster that adds the weight's gradient up itself.  Through Python, where a
// launch takes the host 2 us, 16 rows of 3840 take 5.2 us against 7.5; 32 rows are four for each CTA, and 10.7 against 7.8.
constexpr size_t kTogether = 16;
inline bool together(size_t rows, size_t cols) { return rows <= kTogether && grad_groups(cols); }

// Groups of threads that an SM has: three CTAs of one each, or, where rows are short, more in one CTA of 672 threads (1024 with 64
// registers each took longer).  Groups of several warps have a barrier each, of which there are 15.  Three pieces a thread are for CTAs
// of one group, three an SM: their kernel takes no more threads than one group has (four an SM: 8192 x 3840 65 us, three 57).
inline size_t groups_of_sm(size_t cols) {
    const int pieces = grad_groups(cols), threads = grad_threads(cols);
    if (pieces > 3) return 1;
    if (pieces == 3) return 3;
    return pieces ? std::min(kGradGroupThreads / threads, threads == 32 ? kGradMostGroups : 15) : 3;
}
// as many as run at one time on 148 SMs, two rows at least for each, and not so many that the parts of very long rows outgrow the
// matrices
inline size_t row_groups(size_t rows, size_t cols) {
    return std::min({ceil_div(rows, 2), together(rows, cols) ? 8 : 148 * groups_of_sm(cols), std::max<size_t>(1, (size_t(1) << 28) / cols)});
}
// two rows for each CTA, of one piece a thread
inline bool wide(size_t rows, size_t cols) {
    return cols > size_t(kGradColumns) && cols <= size_t(kGradWide) * 8 && rows <= 2 * row_groups(rows, cols);
}
// Groups of a CTA: all that an SM has where a thread has one piece or those are more than three, which saves parts and their addition.  One CTA of all / CTAs of one,
// us: 30000 x 512 27 / 51, 16384 x 1024 27 / 41, 8192 x 2048 30 / 37; three: 8192 x 3584 47 / 43, 8192 x 5376 80 / 65.
inline size_t groups_of_cta(size_t rows, size_t cols) {
    const bool several = grad_groups(cols) == 1 || groups_of_sm(cols) > 3;
    return together(rows, cols) || wide(rows, cols) || !several ? 1 : ceil_div(row_groups(rows, cols), 148);
}
// CTAs, each with a part of the weight's gradient
inline size_t norm_parts(size_t rows, size_t cols) { return ceil_div(row_groups(rows, cols), groups_of_cta(rows, cols)); }
inline size_t norm_workspace(size_t rows, size_t cols) {
    return together(rows, cols) ? 0 : norm_parts(rows, cols) * part_stride(cols) * sizeof(float);
}

// both are the same matrix: each element is read before it is written by the same thread
inline bool same(const void* p, size_t ldp, const void* q, size_t ldq, size_t rows) { return p == q && (ldp == ldq || rows == 1); }

template <int DT, int W, bool EIGHT>
int launch_norm(const NormArgs& a, cudaStream_t stream) {
    const size_t end = EIGHT ? size_t(a.stages) * 128 : a.cols;
    const int threads = int(std::min<size_t>(kRowThreads, up(ceil_div(end, 8), 32)));
    return launch(end > size_t(kRowThreads) * 8 ? norm_kernel<DT, W, EIGHT, true> : norm_kernel<DT, W, EIGHT, false>, dim3(unsigned(a.rows)),
                  threads, 0, 1, a, stream);
}
template <bool EIGHT>
int launch_norm(const NormArgs& a, int dtype, int width, cudaStream_t stream) {
    if (dtype == EQUARX_BF16)
        return width == 8   ? launch_norm<kBf16, 8, EIGHT>(a, stream)
               : width == 2 ? launch_norm<kBf16, 2, EIGHT>(a, stream)
                            : launch_norm<kBf16, 1, EIGHT>(a, stream);
    return width == 8   ? launch_norm<kFp16, 8, EIGHT>(a, stream)
           : width == 2 ? launch_norm<kFp16, 2, EIGHT>(a, stream)
                        : launch_norm<kFp16, 1, EIGHT>(a, stream);
}

template <int DT, int W, int G, int MOST>
int launch_grad(const NormGradArgs& a, int threads, cudaStream_t stream) {
    // the staged rows (12 bytes a column and more), or the sums in their place
    const size_t sums = a.together || a.groups > 1 ? a.groups * part_stride(a.cols) * sizeof(float) : 0;
    const size_t smem = W == 8 ? size_t(kGradStages) * 3 * 16 * G * threads * a.groups : sums;
    return launch(norm_grad_kernel<DT, W, G, MOST>, dim3(unsigned(a.count)), threads * a.groups, smem, unsigned(a.together), a, stream, true);
}
template <int DT, int W>
int launch_grad(const NormGradArgs& a, cudaStream_t stream) {
    // Rows that are read by elements or pairs do not go through shared memory: more threads with one piece each, and no registers that spill
    // (8191 x 3839: 156 us, with three pieces 215; 8191 x 5375: 224 and 228; by pairs 8191 x 3838: 96 and 126, 8191 x 5374: 145 and 137)
    const bool narrow = W < 8 && a.cols > kGradColumns && a.cols <= kGradWide * 8 && a.groups == 1;
    if (narrow || wide(a.rows, a.cols)) return launch_grad<DT, W, 1, kGradWide>(a, int(up(ceil_div(a.cols, 8), 32)), stream);
    const int threads = grad_threads(a.cols);
    switch (grad_groups(a.cols)) {
        case 1: return launch_grad<DT, W, 1, kGradGroupThreads>(a, threads, stream);
        case 2:
            return groups_of_sm(a.cols) > 3 ? launch_grad<DT, W, 2, kGradGroupThreads>(a, threads, stream)
                                            : launch_grad<DT, W, 2, kGradThreads>(a, threads, stream);
        case 3: return launch_grad<DT, W, 3, kGradThreads>(a, threads, stream);
        case 4: return launch_grad<DT, W, 4, kGradThreads>(a, threads, stream);
        case 5: return launch_grad<DT, W, 5, kGradThreads>(a, threads, stream);
        default: return launch_grad<DT, W, 0, kGradThreads>(a, threads, stream);
    }
}
template <int DT>
int launch_grad(const NormGradArgs& a, int width, cudaStream_t stream) {
    return width == 8 ? launch_grad<DT, 8>(a, stream) : width == 2 ? launch_grad<DT, 2>(a, stream) : launch_grad<DT, 1>(a, stream);
}

// what both outputs share
void set_inputs(NormArgs& a, const void* x, size_t ldx, const void* residual, size_t ldr, const void* weight, int weight_dtype,
                size_t rows, size_t cols, double eps, float offset, void* sum, size_t lds, Access& access) {
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.sum = sum;
    a.ldx = ldx;
    a.ldr = ldr;
    a.lds = lds;
    a.inverse = 1.0 / double(cols);
    a.eps = eps;
    a.offset = offset;
    a.rows = int(rows);
    a.cols = int(cols);
    a.fp32 = weight_dtype == EQUARX_FP32;
    access.add(x, ldx);
    access.add(residual, ldr);
    if (residual) access.add(sum, lds);
    access.add_weight(weight, a.fp32);
}

int check_norm(const void* x, size_t ldx, const void* residual, size_t ldr, const void* weight, int dtype, int weight_dtype,
               size_t rows, size_t cols, double eps, float offset, const void* sum, size_t lds) {
    if (!is_16bit(dtype) || !is_weight(dtype, weight_dtype)) return EQUARX_ERR_FORMAT;
    if (rows > kMaxDim || bad_dim(cols) || bad_ld(ldx, cols) || (residual && (bad_ld(ldr, cols) || bad_ld(lds, cols))))
        return EQUARX_ERR_COUNT;
    if (bad_value(eps, offset)) return EQUARX_ERR_VALUE;
    if (rows == 0) return EQUARX_OK;
    if (!x || !weight || (!residual) != (!sum)) return EQUARX_ERR_NULL;
    if (!aligned(x, 2) || !aligned(residual, 2) || !aligned(sum, 2) || !aligned(weight, size_of(weight_dtype))) return EQUARX_ERR_ALIGN;
    return EQUARX_OK;
}
// the sum against the inputs: it may be one of them
int check_sum(const void* x, size_t ldx, const void* residual, size_t ldr, const void* weight, int weight_dtype, size_t rows,
              size_t cols, const void* sum, size_t lds) {
    if (!residual) return EQUARX_OK;
    const Span s = matrix(sum, rows, cols, lds, 2);
    if (!same(sum, lds, x, ldx, rows) && overlap(s, matrix(x, rows, cols, ldx, 2))) return EQUARX_ERR_ALIAS;
    if (!same(sum, lds, residual, ldr, rows) && overlap(s, matrix(residual, rows, cols, ldr, 2))) return EQUARX_ERR_ALIAS;
    return overlap(s, Span{weight, cols * size_of(weight_dtype)}) ? EQUARX_ERR_ALIAS : EQUARX_OK;
}

}  // namespace

extern "C" {

int equarx_add_rms_norm(const void* x, size_t ldx, const void* residual, size_t ldr, const void* weight, int dtype,
                        int weight_dtype, size_t rows, size_t cols, double eps, float offset, void* sum, size_t lds, void* y,
                        size_t ldy, float* factors, equarx_stream_t stream) {
    TRY(check_norm(x, ldx, residual, ldr, weight, dtype, weight_dtype, rows, cols, eps, offset, sum, lds));
    if (bad_ld(ldy, cols)) return EQUARX_ERR_COUNT;
    if (rows == 0) return EQUARX_OK;
    if (!y) return EQUARX_ERR_NULL;
    if (!aligned(y, 2) || !aligned(factors, 4)) return EQUARX_ERR_ALIGN;
    TRY(check_sum(x, ldx, residual, ldr, weight, weight_dtype, rows, cols, sum, lds));
    TRY(check_overlap({matrix(x, rows, cols, ldx, 2), matrix(residual, rows, cols, ldr, 2), matrix(sum, rows, cols, lds, 2),
                       Span{weight, cols * size_of(weight_dtype)}},
                      {matrix(y, rows, cols, ldy, 2), Span{factors, rows * sizeof(float)}}));
    TRY(check_overlap({}, {matrix(sum, rows, cols, lds, 2), Span{factors, rows * sizeof(float)}}));
    NormArgs a = {};
    Access access;
    set_inputs(a, x, ldx, residual, ldr, weight, weight_dtype, rows, cols, eps, offset, sum, lds, access);
    access.add(y, ldy);
    a.y = y;
    a.ldy = ldy;
    a.factors = factors;
    return launch_norm<false>(a, dtype, access.width(), stream);
}

int equarx_add_rms_norm_fp8(const void* x, size_t ldx, const void* residual, size_t ldr, const void* weight, int dtype,
                            int weight_dtype, size_t rows, size_t cols, double eps, float offset, void* sum, size_t lds,
                            uint8_t* codes, uint8_t* scales, equarx_stream_t stream) {
    TRY(check_norm(x, ldx, residual, ldr, weight, dtype, weight_dtype, rows, cols, eps, offset, sum, lds));
    if (rows == 0) return EQUARX_OK;
    if (!codes || !scales) return EQUARX_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(scales, 16)) return EQUARX_ERR_ALIGN;
    TRY(check_sum(x, ldx, residual, ldr, weight, weight_dtype, rows, cols, sum, lds));
    TRY(check_overlap({matrix(x, rows, cols, ldx, 2), matrix(residual, rows, cols, ldr, 2), matrix(sum, rows, cols, lds, 2),
                       Span{weight, cols * size_of(weight_dtype)}},
                      {Span{codes, rows * fp8_stride(cols)}, Span{scales, equarx_fp8_scales_bytes(rows, cols)}}));
    NormArgs a = {};
    Access access;
    set_inputs(a, x, ldx, residual, ldr, weight, weight_dtype, rows, cols, eps, offset, sum, lds, access);
    a.codes = codes;
    a.scales = scales;
    a.stages = int(fp8_stages(cols));
    return launch_norm<true>(a, dtype, access.width(), stream);
}

size_t equarx_add_rms_norm_backward_workspace_bytes(size_t rows, size_t cols) {
    return rows > kMaxDim || bad_dim(cols) ? 0 : norm_workspace(rows, cols);
}

int equarx_add_rms_norm_backward(const void* dy, size_t lddy, const void* dsum, size_t ldds, const void* sum, size_t lds,
                                 const float* factors, const void* weight, int dtype, int weight_dtype, size_t rows, size_t cols,
                                 float offset, void* dx, size_t lddx, void* dweight, void* workspace, size_t workspace_bytes,
                                 equarx_stream_t stream) {
    if (!is_16bit(dtype) || !is_weight(dtype, weight_dtype)) return EQUARX_ERR_FORMAT;
    if (rows > kMaxDim || bad_dim(cols) || bad_ld(lddy, cols) || (dsum && bad_ld(ldds, cols)) || bad_ld(lds, cols) || bad_ld(lddx, cols))
        return EQUARX_ERR_COUNT;
    if (!std::isfinite(offset)) return EQUARX_ERR_VALUE;
    const size_t size = size_of(weight_dtype), need = dweight ? norm_workspace(rows, cols) : 0;
    if (rows && (!dy || !sum || !factors || !weight || !dx || (need && !workspace))) return EQUARX_ERR_NULL;
    if (rows && workspace_bytes < need) return EQUARX_ERR_WORKSPACE;
    for (const void* p : {dy, dsum, sum, static_cast<const void*>(dx)})
        if (!aligned(p, 2)) return EQUARX_ERR_ALIGN;
    if (!aligned(factors, 4) || !aligned(weight, size) || !aligned(dweight, size) || !aligned(workspace, 16)) return EQUARX_ERR_ALIGN;
    const Span ws{need ? workspace : nullptr, need}, dws{dweight, cols * size};
    TRY(check_overlap({matrix(dy, rows, cols, lddy, 2), matrix(dsum, rows, cols, ldds, 2), matrix(sum, rows, cols, lds, 2),
                       Span{factors, rows * sizeof(float)}, Span{weight, cols * size}},
                      {matrix(dx, rows, cols, lddx, 2), dws, ws}));
    if (rows == 0) {       // a sum over no rows
        cudaError_t e = dweight ? launch_error_to_inject() : cudaSuccess;
        if (e == cudaSuccess && dweight) e = cudaMemsetAsync(dweight, 0, cols * size, stream);
        return e == cudaSuccess ? EQUARX_OK : cuda_failure(e);
    }
    NormGradArgs a = {};
    Access access;
    a.dy = dy;
    a.dsum = dsum;
    a.sum = sum;
    a.factors = factors;
    a.weight = weight;
    a.dx = dx;
    a.dw = dweight;
    a.parts = need ? static_cast<float*>(workspace) : nullptr;
    a.together = dweight && together(rows, cols) ? int(norm_parts(rows, cols)) : 0;
    a.lddy = lddy;
    a.ldds = ldds;
    a.lds = lds;
    a.lddx = lddx;
    a.inverse = float(1.0 / double(cols));
    a.offset = offset;
    a.rows = int(rows);
    a.cols = int(cols);
    a.fp32 = weight_dtype == EQUARX_FP32;
    a.count = int(norm_parts(rows, cols));
    a.groups = int(groups_of_cta(rows, cols));
    access.add(dy, lddy);
    access.add(dsum, ldds);
    access.add(sum, lds);
    access.add(dx, lddx);
    access.add_weight(weight, a.fp32);
    TRY(dtype == EQUARX_BF16 ? launch_grad<kBf16>(a, access.width(), stream) : launch_grad<kFp16>(a, access.width(), stream));
    if (!need) return EQUARX_OK;
    return launch(dtype == EQUARX_BF16 ? norm_parts_kernel<kBf16> : norm_parts_kernel<kFp16>, dim3(unsigned(ceil_div(cols, 32))),
                  kPartsThreads, 0, 1, a, stream, true);
}

}  // extern "C"
