/*
 * na_pyext.c -- a CPython extension that calls na_forward / na_backward of
 * libna.so with the binding's arguments (Python ints for sizes and addresses,
 * a float for the scale), as a cheaper alternative to ctypes' conversion of
 * sixteen or twenty arguments on every call.  It only marshals: the functions
 * are passed in as addresses taken from the library the binding loaded (so
 * NA_LIBRARY keeps selecting the build), nothing is linked, and no torch type
 * is involved.  The binding falls back to ctypes when this module is absent.
 *
 *   forward(fn, rank, extents, kernel_size, dilation, causal, batch, heads,
 *           head_dim, dtype, scale, q, k, v, out, logsumexp, stream) -> status
 *   backward(fn, rank, extents, kernel_size, dilation, causal, batch, heads,
 *            head_dim, dtype, scale, q, k, v, out, logsumexp, dout, dq, dk, dv,
 *            stream) -> status
 *
 *   call(fn, a0, a1, ..) -> status: any function whose arguments are all pointers
 *            or 64-bit integers (at most 16; the entry points of na_seq.h)
 *   metas(t0, t1, ..) -> ((t0.shape, t0.stride(), t0.dtype, t0.device), ..), None for None:
 *            what the binding's checks depend on, the keys of its cached plans
 *
 * Array arguments are the addresses of the problem's int64 / int32 arrays
 * (0 for a NULL causal array); the GIL is released for the call.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "na.h"

typedef na_status (*fwd_fn)(int, const int64_t*, const int32_t*, const int32_t*, const int32_t*,
                            int64_t, int64_t, int64_t, na_dtype, float, const void*, const void*,
                            const void*, void*, float*, na_stream_t);
typedef na_status (*bwd_fn)(int, const int64_t*, const int32_t*, const int32_t*, const int32_t*,
                            int64_t, int64_t, int64_t, na_dtype, float, const void*, const void*,
                            const void*, const void*, const float*, const void*, void*, void*,
                            void*, na_stream_t);

/* The problem arguments shared by both calls: args[1] .. args[10]. */
typedef struct {
    int rank;
    const int64_t* extents;
    const int32_t *ks, *ds, *causal;
    int64_t batch, heads, head_dim;
    na_dtype dtype;
    float scale;
} problem_t;

static int read_problem(PyObject* const* args, problem_t* p) {
    p->rank = (int)PyLong_AsLong(args[1]);
    p->extents = (const int64_t*)PyLong_AsVoidPtr(args[2]);
    p->ks = (const int32_t*)PyLong_AsVoidPtr(args[3]);
    p->ds = (const int32_t*)PyLong_AsVoidPtr(args[4]);
    p->causal = (const int32_t*)PyLong_AsVoidPtr(args[5]);
    p->batch = (int64_t)PyLong_AsLongLong(args[6]);
    p->heads = (int64_t)PyLong_AsLongLong(args[7]);
    p->head_dim = (int64_t)PyLong_AsLongLong(args[8]);
    p->dtype = (na_dtype)PyLong_AsLong(args[9]);
    p->scale = (float)PyFloat_AsDouble(args[10]);
    return PyErr_Occurred() ? -1 : 0;
}

static int read_pointers(PyObject* const* args, Py_ssize_t first, Py_ssize_t n, void** out) {
    for (Py_ssize_t i = 0; i < n; ++i) out[i] = PyLong_AsVoidPtr(args[first + i]);
    return PyErr_Occurred() ? -1 : 0;
}

static PyObject* na_fast_forward(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    (void)self;
    if (nargs != 17) {
        PyErr_SetString(PyExc_TypeError, "forward takes 17 arguments");
        return NULL;
    }
    fwd_fn fn = (fwd_fn)PyLong_AsVoidPtr(args[0]);
    problem_t p;
    void* ptr[6];
    if (PyErr_Occurred() || !fn || read_problem(args, &p) || read_pointers(args, 11, 6, ptr)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "NULL function");
        return NULL;
    }
    na_status st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(p.rank, p.extents, p.ks, p.ds, p.causal, p.batch, p.heads, p.head_dim, p.dtype,
            p.scale, ptr[0], ptr[1], ptr[2], ptr[3], (float*)ptr[4], (na_stream_t)ptr[5]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

static PyObject* na_fast_backward(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    (void)self;
    if (nargs != 21) {
        PyErr_SetString(PyExc_TypeError, "backward takes 21 arguments");
        return NULL;
    }
    bwd_fn fn = (bwd_fn)PyLong_AsVoidPtr(args[0]);
    problem_t p;
    void* ptr[10];
    if (PyErr_Occurred() || !fn || read_problem(args, &p) || read_pointers(args, 11, 10, ptr)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "NULL function");
        return NULL;
    }
    na_status st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(p.rank, p.extents, p.ks, p.ds, p.causal, p.batch, p.heads, p.head_dim, p.dtype,
            p.scale, ptr[0], ptr[1], ptr[2], ptr[3], (const float*)ptr[4], ptr[5], ptr[6], ptr[7],
            ptr[8], (na_stream_t)ptr[9]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

typedef int64_t i64;
typedef na_status (*int_fn)(i64, i64, i64, i64, i64, i64, i64, i64, i64, i64, i64, i64, i64, i64,
                            i64, i64);

static PyObject* na_fast_call(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    (void)self;
    if (nargs < 1 || nargs > 17) {
        PyErr_SetString(PyExc_TypeError, "call takes a function and at most 16 arguments");
        return NULL;
    }
    int_fn fn = (int_fn)PyLong_AsVoidPtr(args[0]);
    /* arguments that the function does not have are passed and not read: on this ABI the
     * caller owns their registers and stack slots */
    i64 a[16] = {0};
    for (Py_ssize_t i = 1; i < nargs && !PyErr_Occurred(); ++i) {
        a[i - 1] = (i64)PyLong_AsLongLong(args[i]);
    }
    if (PyErr_Occurred() || !fn) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "NULL function");
        return NULL;
    }
    na_status st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], a[13],
            a[14], a[15]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

static PyObject* names[4]; /* "shape", "stride", "dtype", "device" */

static PyObject* meta_of(PyObject* t) {
    PyObject* m = PyTuple_New(4);
    if (!m) return NULL;
    for (Py_ssize_t i = 0; i < 4; ++i) {
        PyObject* x = i == 1 ? PyObject_CallMethodNoArgs(t, names[i])
                             : PyObject_GetAttr(t, names[i]);
        if (!x) {
            Py_DECREF(m);
            return NULL;
        }
        PyTuple_SET_ITEM(m, i, x);
    }
    return m;
}

static PyObject* na_fast_metas(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    (void)self;
    PyObject* all = PyTuple_New(nargs);
    if (!all) return NULL;
    for (Py_ssize_t i = 0; i < nargs; ++i) {
        PyObject* m;
        if (args[i] == Py_None) {
            Py_INCREF(Py_None);
            m = Py_None;
        } else if (!(m = meta_of(args[i]))) {
            Py_DECREF(all);
            return NULL;
        }
        PyTuple_SET_ITEM(all, i, m);
    }
    return all;
}

static PyMethodDef methods[] = {
    {"forward", (PyCFunction)(void (*)(void))na_fast_forward, METH_FASTCALL,
     "na_forward through a function address; returns the status"},
    {"backward", (PyCFunction)(void (*)(void))na_fast_backward, METH_FASTCALL,
     "na_backward through a function address; returns the status"},
    {"call", (PyCFunction)(void (*)(void))na_fast_call, METH_FASTCALL,
     "a function of pointers and 64-bit integers through its address; returns the status"},
    {"metas", (PyCFunction)(void (*)(void))na_fast_metas, METH_FASTCALL,
     "shape, strides, type and device of each tensor (None: None)"},
    {NULL, NULL, 0, NULL},
};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_na_fast",
                                    "Argument marshalling for libna.so's hot calls", -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__na_fast(void) {
    static const char* const text[4] = {"shape", "stride", "dtype", "device"};
    for (int i = 0; i < 4; ++i) {
        if (!names[i] && !(names[i] = PyUnicode_InternFromString(text[i]))) return NULL;
    }
    return PyModule_Create(&module);
}
