/* fastcall.c -- the extension module _fast: the training step's entry points of
 * libtda.so called from Python without ctypes' per-argument conversions, which cost
 * more than the launch itself (a lookup of 509 rows, host time: 7.3 us by ctypes with torch's stream
 * object, 2.6 this way).
 *
 * Each function takes its C entry point's arguments in order. A pointer is None, an
 * address or a tensor (its data_ptr()); the stream is None for torch's current stream
 * (the callable given to bind()), an address or a torch stream. The status comes back
 * as an int. bind() receives the entry points' addresses from the library that the
 * package has loaded; nothing is linked here. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/tda.h"

static PyObject *str_data_ptr, *str_cuda_stream, *current_stream, *linear_desc;

static __typeof__(&tda_linear_forward) f_linear_forward;
static __typeof__(&tda_linear_backward) f_linear_backward;
static __typeof__(&tda_embedding_forward) f_embedding_forward;
static __typeof__(&tda_embedding_backward) f_embedding_backward;
static __typeof__(&tda_grad_clip) f_grad_clip;

/* An argument that does not convert leaves a Python error set; the caller looks once, before the call. Until then no
 * Python code runs for the arguments after it, which would turn the error into a SystemError. */
static long long as_int(PyObject *o) { return PyLong_Check(o) || !PyErr_Occurred() ? PyLong_AsLongLong(o) : 0; }
static size_t as_size(PyObject *o) {
    const long long v = as_int(o);
    if (v < 0 && !PyErr_Occurred()) PyErr_SetString(PyExc_OverflowError, "a workspace size is not negative");
    return (size_t)v;
}
static double as_float(PyObject *o) { return PyFloat_Check(o) || !PyErr_Occurred() ? PyFloat_AsDouble(o) : 0; }
static void *as_address(PyObject *o) { return PyLong_AsVoidPtr(o); }

static void *as_ptr(PyObject *o) {
    if (o == Py_None) return NULL;
    if (PyLong_Check(o)) return as_address(o);
    if (PyErr_Occurred()) return NULL;
    PyObject *a = PyObject_CallMethodNoArgs(o, str_data_ptr);
    if (!a) return NULL;
    void *p = as_address(a);
    Py_DECREF(a);
    return p;
}

static void *as_stream(PyObject *o) {
    if (PyLong_Check(o)) return as_address(o);
    if (PyErr_Occurred()) return NULL;
    PyObject *a = o == Py_None ? PyObject_CallNoArgs(current_stream) : PyObject_GetAttr(o, str_cuda_stream);
    if (!a) return NULL;
    void *p = as_address(a);
    Py_DECREF(a);
    return p;
}

/* The address of a ctypes structure or array, by the buffer protocol; b stays held during the call. */
static void *as_struct(PyObject *o, Py_buffer *b) {
    if (o == Py_None) return NULL;
    if (PyObject_GetBuffer(o, b, PyBUF_SIMPLE)) return NULL;
    return b->buf;
}

/* A layer's descriptor: a LinearDesc, nothing else that happens to have a buffer. */
static const tda_linear_desc *as_desc(PyObject *o, Py_buffer *b) {
    if (o != Py_None && !PyObject_TypeCheck(o, (PyTypeObject *)linear_desc)) {
        PyErr_Format(PyExc_TypeError, "the layer is a LinearDesc, not %.100s", Py_TYPE(o)->tp_name);
        return NULL;
    }
    const tda_linear_desc *L = (const tda_linear_desc *)as_struct(o, b);
    if (L && b->len < (Py_ssize_t)sizeof *L) PyErr_SetString(PyExc_TypeError, "the LinearDesc is too short");
    return L;
}

#define ENTRY(name, count)                                                                       \
    static PyObject *name(PyObject *self, PyObject *const *a, Py_ssize_t n) {                    \
        (void)self;                                                                              \
        if (!f_##name) return PyErr_Format(PyExc_RuntimeError, "_fast.bind() has not been called"); \
        if (n != count) return PyErr_Format(PyExc_TypeError, #name " takes %d arguments, got %zd", count, n);
#define I(k) as_int(a[k])
#define P(k) as_ptr(a[k])
/* The library's call, with other threads free to run: it waits where the launch queue is full. */
#define CALL(expr)                              \
    do {                                        \
        Py_BEGIN_ALLOW_THREADS st = (int)(expr); \
        Py_END_ALLOW_THREADS                    \
    } while (0)
#define N(k) as_size(a[k])

ENTRY(embedding_forward, 12)
    const int dt = (int)I(0), it = (int)I(5);
    const void *E = P(1), *tok = P(6);
    const long long ld_e = I(2), V = I(3), d = I(4), cnt = I(7), ld_o = I(10);
    const float scale = (float)as_float(a[8]);
    void *out = P(9), *s = as_stream(a[11]);
    if (PyErr_Occurred()) return NULL;
    int st;
    CALL(f_embedding_forward((tda_dtype)dt, E, ld_e, V, d, (tda_index_type)it, tok, cnt, scale, out, ld_o, s));
    return PyLong_FromLong(st);
}

ENTRY(embedding_backward, 16)
    const int dt = (int)I(0), it = (int)I(5), gt = (int)I(9);
    const void *dout = P(1), *tok = P(6);
    const long long ld_d = I(2), V = I(3), d = I(4), cnt = I(7), ld_e = I(11);
    const size_t wsb = N(14);
    const float scale = (float)as_float(a[8]), beta = (float)as_float(a[12]);
    void *dE = P(10), *ws = P(13), *s = as_stream(a[15]);
    if (PyErr_Occurred()) return NULL;
    int st;
    CALL(f_embedding_backward((tda_dtype)dt, dout, ld_d, V, d, (tda_index_type)it, tok, cnt, scale, (tda_dtype)gt, dE, ld_e,
                              beta, ws, wsb, s));
    return PyLong_FromLong(st);
}

ENTRY(linear_forward, 16)
    Py_buffer b = {0};
    const tda_linear_desc *L = as_desc(a[0], &b);
    const void *X = P(1), *W = P(4), *bias = P(6), *R = P(7);
    const long long ld_x = I(2), M = I(3), ld_w = I(5), ld_r = I(8), ld_y = I(10), ld_z = I(12);
    const size_t wsb = N(14);
    void *Y = P(9), *Z = P(11), *ws = P(13), *s = as_stream(a[15]);
    int st = 0;
    if (!PyErr_Occurred())
        CALL(f_linear_forward(L, X, ld_x, M, W, ld_w, bias, R, ld_r, Y, ld_y, Z, ld_z, ws, wsb, s));
    if (b.obj) PyBuffer_Release(&b);
    return PyErr_Occurred() ? NULL : PyLong_FromLong(st);
}

ENTRY(linear_backward, 22)
    Py_buffer b = {0};
    const tda_linear_desc *L = as_desc(a[0], &b);
    const void *dY = P(1), *Z = P(3), *X = P(6), *W = P(8);
    const long long ld_dy = I(2), ld_z = I(4), M = I(5), ld_x = I(7), ld_w = I(9), ld_b = I(11), ld_dx = I(13),
                    ld_dw = I(15);
    const size_t wsb = N(20);
    void *B = P(10), *dX = P(12), *dW = P(14), *db = P(16), *ws = P(19), *s = as_stream(a[21]);
    const int gt = (int)I(17);
    const float beta = (float)as_float(a[18]);
    int st = 0;
    if (!PyErr_Occurred())
        CALL(f_linear_backward(L, dY, ld_dy, Z, ld_z, M, X, ld_x, W, ld_w, B, ld_b, dX, ld_dx, dW, ld_dw, db, (tda_dtype)gt,
                               beta, ws, wsb, s));
    if (b.obj) PyBuffer_Release(&b);
    return PyErr_Occurred() ? NULL : PyLong_FromLong(st);
}

ENTRY(grad_clip, 7)
    Py_buffer b = {0};
    const tda_tensor_ref *list = (const tda_tensor_ref *)as_struct(a[0], &b);
    const long long count = I(1);
    const size_t wsb = N(5);
    const float most = (float)as_float(a[2]);
    float *norm = (float *)P(3);
    void *ws = P(4), *s = as_stream(a[6]);
    int st = 0;
    if (!PyErr_Occurred()) {
        /* counts past the entry point's own limit are its to refuse */
        if (list && count <= (1LL << 20) && count > (long long)(b.len / (Py_ssize_t)sizeof(tda_tensor_ref)))
            PyErr_SetString(PyExc_ValueError, "grad_clip: more tensors than the list has entries");
        else
            CALL(f_grad_clip(list, count, most, norm, ws, wsb, s));
    }
    if (b.obj) PyBuffer_Release(&b);
    return PyErr_Occurred() ? NULL : PyLong_FromLong(st);
}

/* bind(current_stream, LinearDesc, linear_forward, linear_backward, embedding_forward, embedding_backward, grad_clip) */
static PyObject *bind(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    if (n != 7) return PyErr_Format(PyExc_TypeError, "bind takes 7 arguments, got %zd", n);
    if (!PyType_Check(a[1])) return PyErr_Format(PyExc_TypeError, "bind: LinearDesc is not a type");
    void *f[5];
    for (int i = 0; i < 5; ++i) f[i] = as_address(a[i + 2]);
    if (PyErr_Occurred()) return NULL;
    Py_INCREF(a[0]);
    Py_XSETREF(current_stream, a[0]);
    Py_INCREF(a[1]);
    Py_XSETREF(linear_desc, a[1]);
    f_linear_forward = (__typeof__(f_linear_forward))f[0];
    f_linear_backward = (__typeof__(f_linear_backward))f[1];
    f_embedding_forward = (__typeof__(f_embedding_forward))f[2];
    f_embedding_backward = (__typeof__(f_embedding_backward))f[3];
    f_grad_clip = (__typeof__(f_grad_clip))f[4];
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind),          METHOD(linear_forward),     METHOD(linear_backward),
                                METHOD(embedding_forward), METHOD(embedding_backward), METHOD(grad_clip),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fast(void) {
    str_data_ptr = PyUnicode_InternFromString("data_ptr");
    str_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (!str_data_ptr || !str_cuda_stream) return NULL;
    return PyModule_Create(&module);
}
