// The feed-forward calls of include/equarx.h for torch tensors.
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
void no_gradient(const at::Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(!wants_gradient(t, what), what, " requires a gradient, which 4-bit products do not have: call under ",
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
PyObject* result(int status, const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {
    if (status) return PyLong_FromLong(status);
    PyObject* const o = PyTuple_New(3);
    if (!o) throw python_error();
    PyTuple_SET_ITEM(o, 0, THPVariable_Wrap(a));
    PyTuple_SET_ITEM(o, 1, THPVariable_Wrap(b));
    PyTuple_SET_ITEM(o, 2, THPVariable_Wrap(c));
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
                         {"bind", bind, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_feedforward", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__feedforward(void) { return PyModule_Create(&module); }
