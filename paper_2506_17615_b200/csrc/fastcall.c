/*
 * The feed-forward entry points of include/equarx.h as Python functions of plain integers.
 *
 * ctypes converts an argument in about 0.1 us; with 10 to 25 of them that is a fifth of what a call for a
 * few tokens costs in all.  Here the same conversion takes a few nanoseconds each.  The module knows no
 * library: bind() is given the addresses of the functions that binding.py has loaded.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>
#include <string.h>

#include "../../include/equarx.h"

static struct {
    int (*fp4_quantize)(const void *, int, size_t, size_t, size_t, int, uint8_t *, uint8_t *, float *, equarx_stream_t);
    int (*fp4_dequantize)(const uint8_t *, const uint8_t *, const float *, size_t, size_t, int, void *, int, size_t,
                          equarx_stream_t);
    int (*fp4_matmul)(const uint8_t *, const uint8_t *, const float *, const uint8_t *, const uint8_t *, const float *, size_t,
                      size_t, size_t, int, void *, int, size_t, equarx_stream_t);
    int (*fp4_linear)(const void *, int, size_t, const uint8_t *, const uint8_t *, const float *, size_t, size_t, size_t, int,
                      void *, size_t, void *, size_t, equarx_stream_t);
    int (*fp4_gated)(const void *, int, size_t, const uint8_t *, const uint8_t *, const float *, const uint8_t *,
                     const uint8_t *, const float *, size_t, size_t, size_t, int, int, void *, size_t, void *, size_t,
                     equarx_stream_t);
    int (*gated_forward)(const void *, size_t, const void *, size_t, const void *, size_t, int, size_t, size_t, size_t, int,
                         void *, size_t, void *, void *, size_t, void *, size_t, equarx_stream_t);
    int (*gated_backward)(const void *, size_t, const void *, size_t, const void *, size_t, const void *, size_t, const void *,
                          const void *, size_t, int, size_t, size_t, size_t, int, void *, size_t, void *, size_t, void *, size_t,
                          void *, size_t, equarx_stream_t);
} entry;

#define MAX_ARGS 25

/* exactly n non-negative integers; 0 on success */
static int integers(const char *name, PyObject *const *args, Py_ssize_t given, Py_ssize_t n, unsigned long long *v) {
    if (given != n) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd integers, got %zd", name, n, given);
        return -1;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        v[i] = PyLong_AsUnsignedLongLong(args[i]);
        if (v[i] == (unsigned long long)-1 && PyErr_Occurred()) return -1;
    }
    return 0;
}

#define P(i) ((void *)(uintptr_t)v[i])
#define Z(i) ((size_t)v[i])
#define I(i) (v[i] > INT_MAX ? -1 : (int)v[i]) /* an enumeration: the library refuses -1 */
#define S(i) ((equarx_stream_t)P(i))

#define ENTRY(name, n, ...)                                                                  \
    static PyObject *py_##name(PyObject *self, PyObject *const *args, Py_ssize_t given) {    \
        unsigned long long v[MAX_ARGS];                                                      \
        int status;                                                                          \
        (void)self;                                                                          \
        if (integers(#name, args, given, n, v)) return NULL;                                 \
        if (!entry.name) {                                                                   \
            PyErr_SetString(PyExc_RuntimeError, #name " is not bound");                      \
            return NULL;                                                                     \
        }                                                                                    \
        Py_BEGIN_ALLOW_THREADS                                                               \
        status = entry.name(__VA_ARGS__);                                                    \
        Py_END_ALLOW_THREADS                                                                 \
        return PyLong_FromLong(status);                                                      \
    }

ENTRY(fp4_quantize, 10, P(0), I(1), Z(2), Z(3), Z(4), I(5), P(6), P(7), P(8), S(9))
ENTRY(fp4_dequantize, 10, P(0), P(1), P(2), Z(3), Z(4), I(5), P(6), I(7), Z(8), S(9))
ENTRY(fp4_matmul, 14, P(0), P(1), P(2), P(3), P(4), P(5), Z(6), Z(7), Z(8), I(9), P(10), I(11), Z(12), S(13))
ENTRY(fp4_linear, 15, P(0), I(1), Z(2), P(3), P(4), P(5), Z(6), Z(7), Z(8), I(9), P(10), Z(11), P(12), Z(13), S(14))
ENTRY(fp4_gated, 19, P(0), I(1), Z(2), P(3), P(4), P(5), P(6), P(7), P(8), Z(9), Z(10), Z(11), I(12), I(13), P(14), Z(15),
      P(16), Z(17), S(18))
ENTRY(gated_forward, 19, P(0), Z(1), P(2), Z(3), P(4), Z(5), I(6), Z(7), Z(8), Z(9), I(10), P(11), Z(12), P(13), P(14), Z(15),
      P(16), Z(17), S(18))
ENTRY(gated_backward, 25, P(0), Z(1), P(2), Z(3), P(4), Z(5), P(6), Z(7), P(8), P(9), Z(10), I(11), Z(12), Z(13), Z(14), I(15),
      P(16), Z(17), P(18), Z(19), P(20), Z(21), P(22), Z(23), S(24))

/* bind(name, address) */
static PyObject *py_bind(PyObject *self, PyObject *args) {
    const char *name;
    unsigned long long address;
    (void)self;
    if (!PyArg_ParseTuple(args, "sK", &name, &address)) return NULL;
#define BIND(field)                                       \
    if (!strcmp(name, #field)) {                          \
        *(void **)&entry.field = (void *)(uintptr_t)address; \
        Py_RETURN_NONE;                                   \
    }
    BIND(fp4_quantize)
    BIND(fp4_dequantize)
    BIND(fp4_matmul)
    BIND(fp4_linear)
    BIND(fp4_gated)
    BIND(gated_forward)
    BIND(gated_backward)
#undef BIND
    PyErr_Format(PyExc_ValueError, "no entry point %s", name);
    return NULL;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(fp4_quantize),
                                METHOD(fp4_dequantize),
                                METHOD(fp4_matmul),
                                METHOD(fp4_linear),
                                METHOD(fp4_gated),
                                METHOD(gated_forward),
                                METHOD(gated_backward),
                                {"bind", py_bind, METH_VARARGS, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcall(void) { return PyModule_Create(&module); }
