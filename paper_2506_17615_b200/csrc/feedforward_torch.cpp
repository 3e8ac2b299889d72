// The feed-forward calls of include/equarx.h, and those beside them (norm, adapters), for torch tensors.
//
// A call for a few tokens keeps the GPU busy for 5 to 10 us, and the same marshalling written in Python
// (checks, allocations, ctypes) took as long: here a check costs nanoseconds and an allocation half a
// microsecond.  Nothing is computed: outputs and workspaces are allocated on the tensors' device, the
// library's entry points are called on its current stream, and their status is returned for the caller to
// raise.  The module knows no library: bind() is given the addresses of the functions that binding.py has
// loaded.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/InferenceMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "../../include/equarx.h"

namespace {

#define ENTRIES(X)                       \
    X(fp4_codes_bytes)                   \
    X(fp4_scales_bytes)                  \
    X(fp4_quantize)                      \
    X(fp4_dequantize)                    \
    X(fp4_matmul)                        \
    X(fp4_linear_workspace_bytes)        \
    X(fp4_linear)                        \
    X(fp4_gated)                         \
    X(fp8_codes_bytes)                   \
    X(fp8_scales_bytes)                  \
    X(fp8_quantize)                      \
    X(fp8_dequantize)                    \
    X(fp8_matmul)                        \
    X(fp8_linear_workspace_bytes)        \
    X(fp8_linear)                        \
    X(fp8_gated)                         \
    X(add_rms_norm)                      \
    X(add_rms_norm_fp8)                  \
    X(add_rms_norm_backward_workspace_bytes) \
    X(add_rms_norm_backward)             \
    X(add_adapters)                      \
    X(add_adapters_workspace_bytes)      \
    X(gated_forward_workspace_bytes)     \
    X(gated_forward)                     \
    X(gated_backward_workspace_bytes)    \
    X(gated_backward)

struct {
#define FIELD(name) decltype(&equarx_##name) name;
    ENTRIES(FIELD)
#undef FIELD
} entry;

// ---------------------------------------------------------------- arguments
const at::Tensor& tensor(PyObject* o, const char* what) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), what, " must be a tensor");
    return THPVariable_Unpack(o);
}
// a count or an enumeration; what does not fit is left to the library to refuse
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
int enumeration(PyObject* o) {
    const int64_t v = integer(o);
    return v < 0 || v > INT_MAX ? -1 : int(v);
}
void arguments(Py_ssize_t given, Py_ssize_t wanted) {
    TORCH_CHECK_TYPE(given == wanted, "expected ", wanted, " arguments, got ", given);
}

int dtype_code(at::ScalarType t, const char* what) {
    if (t == at::kBFloat16) return EQUARX_BF16;
    if (t == at::kHalf) return EQUARX_FP16;
    TORCH_CHECK_VALUE(t == at::kFloat, what, " has type ", t);
    return EQUARX_FP32;
}
at::ScalarType scalar_type(int code) {
    TORCH_CHECK_VALUE(code >= 0 && code <= 2, "unknown element type ", code);
    return code == EQUARX_BF16 ? at::kBFloat16 : code == EQUARX_FP16 ? at::kHalf : at::kFloat;
}

struct Matrix {
    const at::Tensor& t;
    void* p;
    size_t rows, cols, ld;
};
Matrix matrix(const at::Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(t.dim() == 2, what, " must be a matrix");
    TORCH_CHECK_VALUE(t.is_cuda(), what, " must be a CUDA tensor");
    const int64_t r = t.size(0), c = t.size(1), ld = t.stride(0);
    TORCH_CHECK_VALUE(t.stride(1) == 1 || c <= 1, what, " must have contiguous columns");
    // any stride, in or out of the library's range, is reported for a single row, which has no next one
    return {t, t.data_ptr(), size_t(r), size_t(c), size_t(r > 1 ? ld : (c + 15) / 16 * 16)};
}
// a matrix that has to be rows x cols, of a type and on the device of `like`
Matrix matrix(const at::Tensor& t, const char* what, size_t rows, size_t cols, at::ScalarType type, const at::Tensor& like) {
    const Matrix m = matrix(t, what);
    TORCH_CHECK_VALUE(m.rows == rows && m.cols == cols && t.scalar_type() == type && t.device() == like.device(), what, " is ",
                      t.sizes(), " ", t.scalar_type(), " on ", t.device(), ", expected [", rows, ", ", cols, "] ", type, " on ",
                      like.device());
    return m;
}
Matrix matrix(const at::Tensor& t, const char* what, size_t rows, size_t cols, const at::Tensor& like) {
    return matrix(t, what, rows, cols, like.scalar_type(), like);
}

// The library knows nothing of autograd, so an output would come back cut off from what made it.
bool wants_gradient(const at::Tensor& t, const char* what) {
    const auto& state = c10::AutogradState::get_tls_state();
    TORCH_CHECK_VALUE(!state.get_fw_grad_mode() || !t._fw_grad(0).defined(), what, " has a forward-mode tangent, which the ",
                      "feed-forward calls do not carry on");
    return state.get_grad_mode() && t.requires_grad();
}
void no_gradient(const at::Tensor& t, const char* what, const char* calls = "4-bit products do") {
    TORCH_CHECK_VALUE(!wants_gradient(t, what), what, " requires a gradient, which ", calls, " not have: call under ",
                      "torch.no_grad(), or with ", what, ".detach()");
}

at::Tensor empty(int64_t rows, int64_t cols, at::ScalarType type, const at::Device& device) {
    return at::detail::empty_cuda({rows, cols}, type, device, c10::nullopt);
}
// nothing is allocated for 0 bytes
at::Tensor bytes(size_t n, const at::Device& device) {
    return n ? at::detail::empty_cuda({int64_t(n)}, at::kByte, device, c10::nullopt) : at::Tensor();
}
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// ---------------------------------------------------------------- 4-bit matrices
// One buffer: scales, row factors (NV), codes, each part starting on a multiple of 256 bytes.
struct Layout {
    size_t row_scales, codes, end;
};
Layout layout(size_t rows, size_t cols, int format) {
    const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    Layout l;
    l.row_scales = up(entry.fp4_scales_bytes(rows, cols, format));
    l.codes = l.row_scales + (format == EQUARX_FP4_NV ? up(rows * 4) : 0);
    l.end = l.codes + entry.fp4_codes_bytes(rows, cols);
    return l;
}
struct Fp4 {
    uint8_t *codes, *scales;
    float* row_scales;
};
Fp4 parts(const at::Tensor& data, size_t rows, size_t cols, int format, const at::Device& device) {
    const Layout l = layout(rows, cols, format);
    TORCH_CHECK_VALUE(data.is_contiguous() && data.scalar_type() == at::kByte && size_t(data.numel()) == l.end,
                      "not the buffer of a ", rows, " x ", cols, " matrix");
    TORCH_CHECK_VALUE(data.device() == device, "the operands are on different devices");
    uint8_t* const p = static_cast<uint8_t*>(data.data_ptr());
    return {p + l.codes, p, format == EQUARX_FP4_NV ? reinterpret_cast<float*>(p + l.row_scales) : nullptr};
}

// ---------------------------------------------------------------- calls
// fn(stream) with the device current and the interpreter lock released
template <typename Call>
int call(const at::Device& device, Call&& fn) {
    const c10::cuda::CUDAGuard guard(device);
    const auto stream = reinterpret_cast<equarx_stream_t>(c10::cuda::getCurrentCUDAStream(device.index()).stream());
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(stream);
    Py_END_ALLOW_THREADS
    return status;
}
PyObject* result(int status, const at::Tensor& t) { return status ? PyLong_FromLong(status) : THPVariable_Wrap(t); }
template <typename... Tensors>
PyObject* result(int status, const at::Tensor& a, const at::Tensor& b, const Tensors&... more) {
    if (status) return PyLong_FromLong(status);
    PyObject* const o = PyTuple_New(2 + sizeof...(more));
    if (!o) throw python_error();
    Py_ssize_t i = 0;
    for (const at::Tensor* t : {&a, &b, &more...}) PyTuple_SET_ITEM(o, i++, THPVariable_Wrap(*t));
    return o;
}

// each returns its tensors, or the library's status as an integer

// quantize(x, format) -> buffer
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 2);
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const int format = enumeration(a[1]), dtype = dtype_code(x.t.scalar_type(), "x");
    const at::Device device = x.t.device();
    const Layout l = layout(x.rows, x.cols, format);
    const at::Tensor data = at::detail::empty_cuda({int64_t(l.end)}, at::kByte, device, c10::nullopt);
    const Fp4 q = parts(data, x.rows, x.cols, format, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.fp4_quantize(x.p, dtype, x.rows, x.cols, x.ld, format, q.codes, q.scales, q.row_scales, s);
    }), data);
    END_HANDLE_TH_ERRORS
}

// dequantize(buffer, rows, cols, format, dtype)
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 5);
    const at::Tensor& data = tensor(a[0], "the matrix");
    const size_t rows = integer(a[1]), cols = integer(a[2]);
    const int format = enumeration(a[3]), dtype = enumeration(a[4]);
    const Fp4 q = parts(data, rows, cols, format, data.device());
    const at::Tensor out = empty(rows, cols, scalar_type(dtype), data.device());
    return result(call(data.device(), [&](equarx_stream_t s) {
        return entry.fp4_dequantize(q.codes, q.scales, q.row_scales, rows, cols, format, out.data_ptr(), dtype, cols, s);
    }), out);
    END_HANDLE_TH_ERRORS
}

// matmul(buffer a, rows of a, buffer b, rows of b, cols, format, dtype)
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 7);
    const at::Tensor &da = tensor(a[0], "a"), &db = tensor(a[2], "b");
    const size_t m = integer(a[1]), rows = integer(a[3]), k = integer(a[4]);
    const int format = enumeration(a[5]), dtype = enumeration(a[6]);
    const Fp4 qa = parts(da, m, k, format, da.device()), qb = parts(db, rows, k, format, da.device());
    const at::Tensor out = empty(m, rows, scalar_type(dtype), da.device());
    return result(call(da.device(), [&](equarx_stream_t s) {
        return entry.fp4_matmul(qa.codes, qa.scales, qa.row_scales, qb.codes, qb.scales, qb.row_scales, m, rows, k, format,
                                out.data_ptr(), dtype, rows, s);
    }), out);
    END_HANDLE_TH_ERRORS
}

// linear(x, buffer w, rows of w, cols, format)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 5);
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const at::Tensor& dw = tensor(a[1], "w");
    const size_t rows = integer(a[2]), k = integer(a[3]);
    const int format = enumeration(a[4]), dtype = dtype_code(x.t.scalar_type(), "x");
    TORCH_CHECK_VALUE(x.cols == k, "x has ", x.cols, " columns, the weight ", k);
    no_gradient(x.t, "x");
    const at::Device device = x.t.device();
    const Fp4 w = parts(dw, rows, k, format, device);
    const at::Tensor out = empty(x.rows, rows, x.t.scalar_type(), device);
    const size_t need = entry.fp4_linear_workspace_bytes(x.rows, k, format);
    const at::Tensor ws = bytes(need, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.fp4_linear(x.p, dtype, x.ld, w.codes, w.scales, w.row_scales, x.rows, rows, k, format, out.data_ptr(), rows,
                                address(ws), need, s);
    }), out);
    END_HANDLE_TH_ERRORS
}

// gated(x, buffer wg, buffer wu, rows, cols, format, act)
PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 7);
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const at::Tensor &dg = tensor(a[1], "wg"), &du = tensor(a[2], "wu");
    const size_t rows = integer(a[3]), k = integer(a[4]);
    const int format = enumeration(a[5]), act = enumeration(a[6]), dtype = dtype_code(x.t.scalar_type(), "x");
    TORCH_CHECK_VALUE(x.cols == k, "x has ", x.cols, " columns, the weights ", k);
    no_gradient(x.t, "x");
    const at::Device device = x.t.device();
    const Fp4 g = parts(dg, rows, k, format, device), u = parts(du, rows, k, format, device);
    const at::Tensor h = empty(x.rows, rows, x.t.scalar_type(), device);
    const size_t need = entry.fp4_linear_workspace_bytes(x.rows, k, format);
    const at::Tensor ws = bytes(need, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.fp4_gated(x.p, dtype, x.ld, g.codes, g.scales, g.row_scales, u.codes, u.scales, u.row_scales, x.rows, rows,
                               k, format, act, h.data_ptr(), rows, address(ws), need, s);
    }), h);
    END_HANDLE_TH_ERRORS
}

// gated_forward(x, wg, wu, act, save, g and u in fp32); None, and nothing is done, where autograd wants gradients
PyObject* gated_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 6);
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const at::Tensor& tg = tensor(a[1], "wg");
    const size_t f = tg.dim() ? size_t(tg.size(0)) : 0;
    const Matrix wg = matrix(tg, "wg", f, x.cols, x.t), wu = matrix(tensor(a[2], "wu"), "wu", f, x.cols, x.t);
    const int act = enumeration(a[3]), save = PyObject_IsTrue(a[4]), wide = PyObject_IsTrue(a[5]),
              dtype = dtype_code(x.t.scalar_type(), "x") | (wide ? EQUARX_KEPT_FP32 : 0);
    if (save < 0 || wide < 0) throw python_error();
    const bool grad[] = {wants_gradient(x.t, "x"), wants_gradient(wg.t, "wg"), wants_gradient(wu.t, "wu")};
    if (grad[0] || grad[1] || grad[2]) Py_RETURN_NONE;
    const at::Device device = x.t.device();
    const at::Tensor h = empty(x.rows, f, x.t.scalar_type(), device);
    at::Tensor g, u;
    if (save) {
        const at::ScalarType kept = wide ? at::kFloat : x.t.scalar_type();
        g = empty(x.rows, f, kept, device);
        u = empty(x.rows, f, kept, device);
    }
    const size_t need = entry.gated_forward_workspace_bytes(x.rows, f, x.cols, x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld);
    const at::Tensor ws = bytes(need, device);
    const int status = call(device, [&](equarx_stream_t s) {
        return entry.gated_forward(x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, dtype, x.rows, f, x.cols, act, h.data_ptr(), f, address(g),
                                   address(u), f, address(ws), need, s);
    });
    return save ? result(status, h, g, u) : result(status, h);
    END_HANDLE_TH_ERRORS
}

// gated_backward(dh, x, wg, wu, g, u, act)
PyObject* gated_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 7);
    const Matrix x = matrix(tensor(a[1], "x"), "x");
    const at::Tensor& tg = tensor(a[2], "wg");
    const size_t m = x.rows, k = x.cols, f = tg.dim() ? size_t(tg.size(0)) : 0;
    const Matrix wg = matrix(tg, "wg", f, k, x.t), wu = matrix(tensor(a[3], "wu"), "wu", f, k, x.t);
    const at::Tensor& kept = tensor(a[4], "g");
    const bool wide = kept.scalar_type() == at::kFloat;
    const at::ScalarType type = wide ? at::kFloat : x.t.scalar_type();
    const Matrix dh = matrix(tensor(a[0], "dh"), "dh", m, f, x.t), g = matrix(kept, "g", m, f, type, x.t),
                 u = matrix(tensor(a[5], "u"), "u", m, f, type, x.t);
    TORCH_CHECK_VALUE(g.ld == u.ld, "g and u have different row strides");
    const int act = enumeration(a[6]), dtype = dtype_code(x.t.scalar_type(), "x") | (wide ? EQUARX_KEPT_FP32 : 0);
    const at::Device device = x.t.device();
    const at::Tensor dx = empty(m, k, x.t.scalar_type(), device), dwg = empty(f, k, x.t.scalar_type(), device),
                     dwu = empty(f, k, x.t.scalar_type(), device);
    const size_t need = entry.gated_backward_workspace_bytes(m, f, k, x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld);
    const at::Tensor ws = bytes(need, device);
    const int status = call(device, [&](equarx_stream_t s) {
        return entry.gated_backward(dh.p, dh.ld, x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, g.p, u.p, g.ld, dtype, m, f, k, act,
                                    dx.data_ptr(), k, dwg.data_ptr(), k, dwu.data_ptr(), k, address(ws), need, s);
    });
    return result(status, dx, dwg, dwu);
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- 8-bit matrices
// One buffer: scales, then codes from a multiple of 256 bytes on.
struct Fp8 {
    uint8_t *codes, *scales;
};
size_t fp8_codes_at(size_t rows, size_t cols) { return (entry.fp8_scales_bytes(rows, cols) + 255) / 256 * 256; }
size_t fp8_bytes(size_t rows, size_t cols) { return fp8_codes_at(rows, cols) + entry.fp8_codes_bytes(rows, cols); }
Fp8 parts8(const at::Tensor& data, size_t rows, size_t cols, const at::Device& device) {
    TORCH_CHECK_VALUE(data.is_contiguous() && data.scalar_type() == at::kByte && size_t(data.numel()) == fp8_bytes(rows, cols),
                      "not the buffer of a ", rows, " x ", cols, " matrix");
    TORCH_CHECK_VALUE(data.device() == device, "the operands are on different devices");
    uint8_t* const p = static_cast<uint8_t*>(data.data_ptr());
    return {p + fp8_codes_at(rows, cols), p};
}
at::Tensor empty8(size_t rows, size_t cols, const at::Device& device) {
    return at::detail::empty_cuda({int64_t(fp8_bytes(rows, cols))}, at::kByte, device, c10::nullopt);
}
constexpr const char* kEight = "8-bit products do";

// quantize8(x) -> buffer
PyObject* quantize8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 1);
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const int dtype = dtype_code(x.t.scalar_type(), "x");
    const at::Device device = x.t.device();
    const at::Tensor data = empty8(x.rows, x.cols, device);
    const Fp8 q = parts8(data, x.rows, x.cols, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.fp8_quantize(x.p, dtype, x.rows, x.cols, x.ld, q.codes, q.scales, s);
    }), data);
    END_HANDLE_TH_ERRORS
}

// dequantize8(buffer, rows, cols, dtype)
PyObject* dequantize8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 4);
    const at::Tensor& data = tensor(a[0], "the matrix");
    const size_t rows = integer(a[1]), cols = integer(a[2]);
    const int dtype = enumeration(a[3]);
    const Fp8 q = parts8(data, rows, cols, data.device());
    const at::Tensor out = empty(rows, cols, scalar_type(dtype), data.device());
    return result(call(data.device(), [&](equarx_stream_t s) {
        return entry.fp8_dequantize(q.codes, q.scales, rows, cols, out.data_ptr(), dtype, cols, s);
    }), out);
    END_HANDLE_TH_ERRORS
}

// matmul8(buffer a, rows of a, buffer b, rows of b, cols, dtype)
PyObject* matmul8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 6);
    const at::Tensor &da = tensor(a[0], "a"), &db = tensor(a[2], "b");
    const size_t m = integer(a[1]), rows = integer(a[3]), k = integer(a[4]);
    const int dtype = enumeration(a[5]);
    const Fp8 qa = parts8(da, m, k, da.device()), qb = parts8(db, rows, k, da.device());
    const at::Tensor out = empty(m, rows, scalar_type(dtype), da.device());
    return result(call(da.device(), [&](equarx_stream_t s) {
        return entry.fp8_matmul(qa.codes, qa.scales, qb.codes, qb.scales, m, rows, k, out.data_ptr(), dtype, rows, s);
    }), out);
    END_HANDLE_TH_ERRORS
}

// gated8(buffer x, rows of x, buffer wg, buffer wu, rows, cols, act, dtype)
PyObject* gated8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 8);
    const at::Tensor &dx = tensor(a[0], "x"), &dg = tensor(a[2], "wg"), &du = tensor(a[3], "wu");
    const size_t m = integer(a[1]), rows = integer(a[4]), k = integer(a[5]);
    const int act = enumeration(a[6]), dtype = enumeration(a[7]);
    const at::Device device = dx.device();
    const Fp8 x = parts8(dx, m, k, device), g = parts8(dg, rows, k, device), u = parts8(du, rows, k, device);
    const at::Tensor h = empty(m, rows, scalar_type(dtype), device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.fp8_gated(x.codes, x.scales, g.codes, g.scales, u.codes, u.scales, m, rows, k, act, h.data_ptr(), dtype, rows, s);
    }), h);
    END_HANDLE_TH_ERRORS
}

// linear8(x, buffer w, rows of w, cols): x quantized in the call
PyObject* linear8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 4);
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const at::Tensor& dw = tensor(a[1], "w");
    const size_t rows = integer(a[2]), k = integer(a[3]);
    const int dtype = dtype_code(x.t.scalar_type(), "x");
    TORCH_CHECK_VALUE(dtype != EQUARX_FP32, "x has 32 bits: activations have 16");
    TORCH_CHECK_VALUE(x.cols == k, "x has ", x.cols, " columns, the weight ", k);
    no_gradient(x.t, "x", kEight);
    const at::Device device = x.t.device();
    const Fp8 w = parts8(dw, rows, k, device);
    const at::Tensor out = empty(x.rows, rows, x.t.scalar_type(), device);
    const size_t need = entry.fp8_linear_workspace_bytes(x.rows, k);
    const at::Tensor ws = bytes(need, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.fp8_linear(x.p, dtype, x.ld, w.codes, w.scales, x.rows, rows, k, out.data_ptr(), rows, address(ws), need, s);
    }), out);
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- norm
struct Vector {
    const at::Tensor& t;
    void* p;
};
Vector vector(const at::Tensor& t, const char* what, size_t size, const at::Tensor& like) {
    TORCH_CHECK_VALUE(t.dim() == 1 && size_t(t.size(0)) == size && t.is_contiguous() && t.device() == like.device(), what, " is ",
                      t.sizes(), " on ", t.device(), ", expected [", size, "], contiguous, on ", like.device());
    return {t, t.data_ptr()};
}
// of the matrices' type or fp32
int weight_code(const at::Tensor& t, const at::Tensor& like) {
    TORCH_CHECK_VALUE(t.scalar_type() == like.scalar_type() || t.scalar_type() == at::kFloat, "weight has type ", t.scalar_type(),
                      ", expected ", like.scalar_type(), " or ", at::kFloat);
    return dtype_code(t.scalar_type(), "weight");
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
struct Norm {
    Matrix x;
    const void* residual;
    size_t ldr;
    Vector weight;
    int dtype, weight_dtype;
    double eps;
    float offset;
    at::Tensor sum;          // x itself where there is no residual
    void* psum;
    bool gradient;
};
// x, residual or None, weight, eps, offset
Norm norm_arguments(PyObject* const* a) {
    const Matrix x = matrix(tensor(a[0], "x"), "x");
    const bool add = a[1] != Py_None;
    const Vector w = vector(tensor(a[2], "weight"), "weight", x.cols, x.t);
    Norm m{x, nullptr, 0, w, dtype_code(x.t.scalar_type(), "x"), weight_code(w.t, x.t), number(a[3]), float(number(a[4])), x.t, nullptr,
           false};
    m.gradient = wants_gradient(x.t, "x");
    m.gradient |= wants_gradient(w.t, "weight");
    if (add) {
        const Matrix r = matrix(tensor(a[1], "residual"), "residual", x.rows, x.cols, x.t);
        m.gradient |= wants_gradient(r.t, "residual");
        m.residual = r.p;
        m.ldr = r.ld;
    }
    return m;
}
void allocate_sum(Norm& m) {
    if (!m.ldr) return;
    m.sum = empty(m.x.rows, m.x.cols, m.x.t.scalar_type(), m.x.t.device());
    m.psum = m.sum.data_ptr();
}

// add_rms_norm(x, residual, weight, eps, offset, save) -> y, sum, factors with save; None, and nothing is done, where autograd
// wants gradients
PyObject* add_rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 6);
    Norm m = norm_arguments(a);
    const int save = PyObject_IsTrue(a[5]);
    if (save < 0) throw python_error();
    if (m.gradient) Py_RETURN_NONE;
    allocate_sum(m);
    const at::Device device = m.x.t.device();
    const at::Tensor y = empty(m.x.rows, m.x.cols, m.x.t.scalar_type(), device);
    const at::Tensor factors = save ? at::detail::empty_cuda({int64_t(m.x.rows)}, at::kFloat, device, c10::nullopt) : at::Tensor();
    const int status = call(device, [&](equarx_stream_t s) {
        return entry.add_rms_norm(m.x.p, m.x.ld, m.residual, m.ldr, m.weight.p, m.dtype, m.weight_dtype, m.x.rows, m.x.cols, m.eps,
                                  m.offset, m.psum, m.x.cols, y.data_ptr(), m.x.cols, static_cast<float*>(address(factors)), s);
    });
    return save ? result(status, y, m.sum, factors) : result(status, y, m.sum);
    END_HANDLE_TH_ERRORS
}

// add_rms_norm_fp8(x, residual, weight, eps, offset) -> buffer, sum
PyObject* add_rms_norm_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 5);
    Norm m = norm_arguments(a);
    TORCH_CHECK_VALUE(!m.gradient, "an input requires a gradient, which 8-bit outputs do not have: call under torch.no_grad()");
    allocate_sum(m);
    const at::Device device = m.x.t.device();
    const at::Tensor data = empty8(m.x.rows, m.x.cols, device);
    const Fp8 q = parts8(data, m.x.rows, m.x.cols, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.add_rms_norm_fp8(m.x.p, m.x.ld, m.residual, m.ldr, m.weight.p, m.dtype, m.weight_dtype, m.x.rows, m.x.cols, m.eps,
                                      m.offset, m.psum, m.x.cols, q.codes, q.scales, s);
    }), data, m.sum);
    END_HANDLE_TH_ERRORS
}

// add_rms_norm_backward(dy, dsum or None, sum, factors, weight, offset) -> dx, dweight
PyObject* add_rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 6);
    const Matrix sum = matrix(tensor(a[2], "sum"), "sum");
    const Matrix dy = matrix(tensor(a[0], "dy"), "dy", sum.rows, sum.cols, sum.t);
    const void* dsum = nullptr;
    size_t ldds = 0;
    if (a[1] != Py_None) {
        const Matrix d = matrix(tensor(a[1], "dsum"), "dsum", sum.rows, sum.cols, sum.t);
        dsum = d.p;
        ldds = d.ld;
    }
    const Vector factors = vector(tensor(a[3], "factors"), "factors", sum.rows, sum.t);
    TORCH_CHECK_VALUE(factors.t.scalar_type() == at::kFloat, "factors have type ", factors.t.scalar_type());
    const Vector w = vector(tensor(a[4], "weight"), "weight", sum.cols, sum.t);
    const int dtype = dtype_code(sum.t.scalar_type(), "sum"), weight_dtype = weight_code(w.t, sum.t);
    const float offset = float(number(a[5]));
    const at::Device device = sum.t.device();
    const at::Tensor dx = empty(sum.rows, sum.cols, sum.t.scalar_type(), device);
    const at::Tensor dw = at::detail::empty_cuda({int64_t(sum.cols)}, w.t.scalar_type(), device, c10::nullopt);
    const size_t need = entry.add_rms_norm_backward_workspace_bytes(sum.rows, sum.cols);
    const at::Tensor ws = bytes(need, device);
    return result(call(device, [&](equarx_stream_t s) {
        return entry.add_rms_norm_backward(dy.p, dy.ld, dsum, ldds, sum.p, sum.ld, static_cast<const float*>(factors.p), w.p, dtype,
                                           weight_dtype, sum.rows, sum.cols, offset, dx.data_ptr(), sum.cols, dw.data_ptr(),
                                           address(ws), need, s);
    }), dx, dw);
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- adapters
// add_adapters(y, x, a, b, index, scale or None, out or None)
PyObject* add_adapters(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    arguments(count, 7);
    const Matrix y = matrix(tensor(args[0], "y"), "y");
    const at::Tensor &tx = tensor(args[1], "x"), &ta = tensor(args[2], "a"), &tb = tensor(args[3], "b");
    const size_t k = tx.dim() == 2 ? tx.size(1) : 0, n = y.cols, m = y.rows;
    const Matrix x = matrix(tx, "x", m, k, y.t);
    TORCH_CHECK_VALUE(ta.dim() == 3 && tb.dim() == 3, "a and b must be [adapters, rank, k] and [adapters, n, rank]");
    const int64_t adapters = ta.size(0), rank = ta.size(1);
    for (const at::Tensor* t : {&ta, &tb})
        TORCH_CHECK_VALUE(t->is_contiguous() && t->scalar_type() == y.t.scalar_type() && t->device() == y.t.device(),
                          "a and b must be contiguous, of y's type and on its device");
    TORCH_CHECK_VALUE(size_t(ta.size(2)) == k && tb.size(0) == adapters && size_t(tb.size(1)) == n && tb.size(2) == rank, "a is ",
                      ta.sizes(), " and b ", tb.sizes(), ", expected [", adapters, ", ", rank, ", ", k, "] and [", adapters, ", ", n,
                      ", ", rank, "]");
    const Vector index = vector(tensor(args[4], "index"), "index", m, y.t);
    TORCH_CHECK_VALUE(index.t.scalar_type() == at::kInt, "index has type ", index.t.scalar_type(), ", expected ", at::kInt);
    const float* scale = nullptr;
    constexpr const char* calls = "adapters of many requests do";
    if (args[5] != Py_None) {
        const Vector v = vector(tensor(args[5], "scale"), "scale", adapters, y.t);
        TORCH_CHECK_VALUE(v.t.scalar_type() == at::kFloat, "scale has type ", v.t.scalar_type(), ", expected ", at::kFloat);
        no_gradient(v.t, "scale", calls);
        scale = static_cast<const float*>(v.p);
    }
    no_gradient(y.t, "y", calls);
    no_gradient(tx, "x", calls);
    no_gradient(ta, "a", calls);
    no_gradient(tb, "b", calls);
    const int dtype = dtype_code(y.t.scalar_type(), "y");
    const at::Device device = y.t.device();
    const at::Tensor out = args[6] == Py_None ? empty(m, n, y.t.scalar_type(), device) : tensor(args[6], "out");
    const Matrix o = matrix(out, "out", m, n, y.t);
    no_gradient(out, "out", calls);
    TORCH_CHECK(!out.is_inference() || c10::InferenceMode::is_enabled(), "out is an inference tensor: it is written in inference mode only");
    const size_t need = entry.add_adapters_workspace_bytes(m, n, k, rank, adapters);
    const at::Tensor ws = bytes(need, device);
    const int status = call(device, [&](equarx_stream_t s) {
        return entry.add_adapters(y.p, y.ld, x.p, x.ld, ta.data_ptr(), tb.data_ptr(), static_cast<const int32_t*>(index.p), scale, dtype, m,
                                  n, k, rank, adapters, o.p, o.ld, address(ws), need, s);
    });
    // what autograd has saved of a caller's tensor is not what it was, whatever the gradient mode is now
    if (!status && args[6] != Py_None) out.unsafeGetTensorImpl()->bump_version();
    return result(status, out);
    END_HANDLE_TH_ERRORS
}

// layout8(rows, cols) -> offset of the codes, size
PyObject* layout8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 2);
    const size_t rows = integer(a[0]), cols = integer(a[1]);
    return Py_BuildValue("nn", Py_ssize_t(fp8_codes_at(rows, cols)), Py_ssize_t(fp8_bytes(rows, cols)));
    END_HANDLE_TH_ERRORS
}

// layout(rows, cols, format) -> offset of the row factors, offset of the codes, size
PyObject* layout_of(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 3);
    const Layout l = layout(integer(a[0]), integer(a[1]), enumeration(a[2]));
    return Py_BuildValue("nnn", Py_ssize_t(l.row_scales), Py_ssize_t(l.codes), Py_ssize_t(l.end));
    END_HANDLE_TH_ERRORS
}

// bind(name, address)
PyObject* bind(PyObject*, PyObject* args) {
    const char* name;
    unsigned long long where;
    if (!PyArg_ParseTuple(args, "sK", &name, &where)) return nullptr;
#define BIND(field)                                                      \
    if (!std::strcmp(name, #field)) {                                    \
        entry.field = reinterpret_cast<decltype(entry.field)>(where);    \
        Py_RETURN_NONE;                                                  \
    }
    ENTRIES(BIND)
#undef BIND
    PyErr_Format(PyExc_ValueError, "no entry point %s", name);
    return nullptr;
}

#define METHOD(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD("quantize", quantize),
                         METHOD("dequantize", dequantize),
                         METHOD("matmul", matmul),
                         METHOD("linear", linear),
                         METHOD("gated", gated),
                         METHOD("gated_forward", gated_forward),
                         METHOD("gated_backward", gated_backward),
                         METHOD("layout", layout_of),
                         METHOD("quantize8", quantize8),
                         METHOD("dequantize8", dequantize8),
                         METHOD("matmul8", matmul8),
                         METHOD("linear8", linear8),
                         METHOD("gated8", gated8),
                         METHOD("layout8", layout8),
                         METHOD("add_rms_norm", add_rms_norm),
                         METHOD("add_rms_norm_fp8", add_rms_norm_fp8),
                         METHOD("add_rms_norm_backward", add_rms_norm_backward),
                         METHOD("add_adapters", add_adapters),
                         {"bind", bind, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_feedforward", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__feedforward(void) { return PyModule_Create(&module); }
