// The binding's calls that a decode step makes most often, compiled: fbq_linear, and below it fbq_attention and fbq_cache_append.
//
// The binding's call of fbq_linear for one layer whose result and workspace the caller keeps: collects the pointers of the tensors and calls the
// library, without the argument objects that ctypes builds (one token through 4096 x 4096: the call took longer than its kernel, 6.1 us; 5.0 this way).
// It knows nothing of torch: it asks the objects what the binding's Python code asks (is_cuda, is_contiguous(), data_ptr(), numel(),
// element_size()).  Whatever is not as it should be makes it return None, and the Python code does the call, or raises;
// exceptions that are no `Exception` pass through.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "fbq.h"

typedef fbq_status (*linear_fn)(const fbq_desc *, int, const void *, const void *, const void *, const void *, const void *, const void *, void *, void *,
                                size_t, fbq_stream);

static PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_numel, *s_element_size, *s_desc, *s_N, *s_K, *s_r, *s_bits, *s_group, *s_shape, *s_dtype, *s_stride;
static PyObject *s_tensor[5];                           // qweight, scales, zeros, At, Bt

// An attribute or a method's result as a whole number; 0 where it is none.
static int number(PyObject *v, unsigned long long *out)
{
    const int ok = v && PyLong_CheckExact(v);
    if (ok) *out = PyLong_AsUnsignedLongLongMask(v);
    Py_XDECREF(v);
    return ok;
}

static int is_true(PyObject *v)
{
    const int yes = v == Py_True;
    Py_XDECREF(v);
    return yes;
}

static int pointer(PyObject *t, unsigned long long *out)
{
    *out = 0;
    if (t == Py_None) return 1;
    return is_true(PyObject_GetAttr(t, s_is_cuda)) && is_true(PyObject_CallMethodNoArgs(t, s_is_contiguous)) && number(PyObject_CallMethodNoArgs(t, s_data_ptr), out);
}

// linear(address of fbq_linear, layer, x, y, workspace, stream) -> status, or None
static PyObject *linear(PyObject *self, PyObject *const *arg, Py_ssize_t n)
{
    (void)self;
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "six arguments");
        return NULL;
    }
    unsigned long long fn, p[8] = {0}, field[5], M = 0, count = 0, each = 0, stream;
    PyObject *const names[5] = {s_N, s_K, s_r, s_bits, s_group};
    PyObject *desc = NULL, *shape = NULL, *first = NULL;
    int ok = PyLong_CheckExact(arg[0]) && PyLong_CheckExact(arg[5]);
    fn = ok ? PyLong_AsUnsignedLongLongMask(arg[0]) : 0;
    stream = ok ? PyLong_AsUnsignedLongLongMask(arg[5]) : 0;
    ok = ok && fn && (desc = PyObject_GetAttr(arg[1], s_desc));
    for (int i = 0; ok && i < 5; ++i) ok = number(PyObject_GetAttr(desc, names[i]), &field[i]) && field[i] <= INT32_MAX;
    Py_XDECREF(desc);
    ok = ok && (shape = PyObject_GetAttr(arg[2], s_shape)) && (first = PySequence_GetItem(shape, 0)) && PyLong_CheckExact(first);
    if (ok) M = PyLong_AsUnsignedLongLongMask(first);
    Py_XDECREF(first);
    Py_XDECREF(shape);
    ok = ok && M <= INT32_MAX && pointer(arg[2], &p[0]);
    for (int i = 0; ok && i < 5; ++i) {
        PyObject *t = PyObject_GetAttr(arg[1], s_tensor[i]);
        ok = t && pointer(t, &p[1 + i]);
        Py_XDECREF(t);
    }
    ok = ok && pointer(arg[3], &p[6]) && pointer(arg[4], &p[7]);
    if (ok && arg[4] != Py_None) ok = number(PyObject_CallMethodNoArgs(arg[4], s_numel), &count) && number(PyObject_CallMethodNoArgs(arg[4], s_element_size), &each);
    if (!ok) {
        if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return NULL;   // (an interrupt, say: not this call's to drop)
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const fbq_desc d = {(int32_t)field[0], (int32_t)field[1], (int32_t)field[2], (int32_t)field[3], (int32_t)field[4]};
    fbq_status st;
    Py_BEGIN_ALLOW_THREADS                              // (as ctypes does)
    st = ((linear_fn)(uintptr_t)fn)(&d, (int)M, (const void *)(uintptr_t)p[0], (const void *)(uintptr_t)p[1], (const void *)(uintptr_t)p[2],
                                    (const void *)(uintptr_t)p[3], (const void *)(uintptr_t)p[4], (const void *)(uintptr_t)p[5],
                                    (void *)(uintptr_t)p[6], (void *)(uintptr_t)p[7], (size_t)(count * each), (fbq_stream)(uintptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

// What attention and append ask of a tensor: [T, heads, head_dim] on the device, of one type, a token's heads in one piece.
typedef struct { unsigned long long at; long long T, heads, dim, stride; } tokens_t;

static int whole(PyObject *tuple, int n, long long *out)
{
    int ok = tuple && PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == n;
    for (int i = 0; ok && i < n; ++i) {
        PyObject *v = PyTuple_GET_ITEM(tuple, i);
        ok = PyLong_CheckExact(v);
        if (ok) out[i] = PyLong_AsLongLong(v);
    }
    Py_XDECREF(tuple);
    return ok && !PyErr_Occurred();
}

static int is_of(PyObject *t, PyObject *dtype)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    Py_XDECREF(d);
    return d == dtype;
}

static int tokens(PyObject *t, PyObject *dtype, tokens_t *x)
{
    long long shape[3], stride[3];
    if (!is_of(t, dtype) || !whole(PyObject_GetAttr(t, s_shape), 3, shape) || !whole(PyObject_CallMethodNoArgs(t, s_stride), 3, stride) || stride[2] != 1 ||
        (stride[1] != shape[2] && shape[1] > 1) || !is_true(PyObject_GetAttr(t, s_is_cuda)) || !number(PyObject_CallMethodNoArgs(t, s_data_ptr), &x->at))
        return 0;
    x->T = shape[0]; x->heads = shape[1]; x->dim = shape[2];
    x->stride = shape[0] > 1 ? stride[0] : shape[1] * shape[2];
    return 1;
}

// A contiguous device tensor of the type, `n` elements where that is not negative; None: a null pointer.
static int list(PyObject *t, PyObject *dtype, long long n, unsigned long long *at, unsigned long long *count)
{
    *at = 0;
    *count = 0;
    if (t == Py_None) return 1;
    return is_of(t, dtype) && pointer(t, at) && number(PyObject_CallMethodNoArgs(t, s_numel), count) && (n < 0 || (long long)*count == n);
}

static int whole_number(PyObject *v, unsigned long long *out)
{
    if (!PyLong_CheckExact(v)) return 0;
    *out = PyLong_AsUnsignedLongLongMask(v);
    return 1;
}

static PyObject *not_as_expected(void)
{
    if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return NULL;   // (an interrupt, say: not this call's to drop)
    PyErr_Clear();
    Py_RETURN_NONE;
}

typedef fbq_status (*attention_fn)(const fbq_attention_call *, void *, size_t, fbq_stream);

// attention(address of fbq_attention, address of the fbq_cache, its type, int32, float32, layer, q, q_start, max_q, shared, scale, out, lse, workspace, stream) -> status, or None
static PyObject *attention(PyObject *self, PyObject *const *arg, Py_ssize_t n)
{
    (void)self;
    if (n != 15) {
        PyErr_SetString(PyExc_TypeError, "fifteen arguments");
        return NULL;
    }
    unsigned long long fn, cache, layer, max_q, stream, q_start, shared, lse, ws, count, each = 0;
    tokens_t q, out;
    if (!whole_number(arg[0], &fn) || !whole_number(arg[1], &cache) || !fn || !cache) return not_as_expected();
    fbq_attention_call c;
    c.cache = *(const fbq_cache *)(uintptr_t)cache;
    int ok = whole_number(arg[5], &layer) && layer <= INT32_MAX && whole_number(arg[8], &max_q) && max_q <= INT32_MAX && whole_number(arg[14], &stream) && PyFloat_CheckExact(arg[10]);
    ok = ok && tokens(arg[6], arg[2], &q) && tokens(arg[11], arg[2], &out) && q.T == out.T && q.heads == out.heads && q.dim == out.dim && q.dim == c.cache.desc.head_dim &&
         q.T <= INT32_MAX && q.heads <= INT32_MAX;
    ok = ok && list(arg[7], arg[3], c.cache.rows + 1LL, &q_start, &count) && list(arg[12], arg[4], q.T * q.heads, &lse, &count) && list(arg[9], arg[3], -1, &shared, &count) &&
         count <= INT32_MAX;
    if (ok) c.n_shared = (int32_t)count;
    if (ok && lse) {
        long long shape[2];
        ok = whole(PyObject_GetAttr(arg[12], s_shape), 2, shape) && shape[0] == q.T && shape[1] == q.heads;
    }
    ok = ok && pointer(arg[13], &ws);                       // (no workspace: the library says whether the call needs one)
    count = 0;
    if (ok && arg[13] != Py_None) ok = number(PyObject_CallMethodNoArgs(arg[13], s_numel), &count) && number(PyObject_CallMethodNoArgs(arg[13], s_element_size), &each);
    if (!ok) return not_as_expected();
    c.layer = (int32_t)layer; c.heads = (int32_t)q.heads; c.T = (int32_t)q.T; c.max_q = (int32_t)max_q;
    c.q_start = (const int32_t *)(uintptr_t)q_start;
    c.q = (const void *)(uintptr_t)q.at; c.q_stride = q.stride;
    c.out = (void *)(uintptr_t)out.at; c.out_stride = out.stride;
    c.lse = (float *)(uintptr_t)lse;
    c.shared = (const int32_t *)(uintptr_t)shared;
    c.scale = (float)PyFloat_AS_DOUBLE(arg[10]);
    fbq_status st;
    Py_BEGIN_ALLOW_THREADS
    st = ((attention_fn)(uintptr_t)fn)(&c, (void *)(uintptr_t)ws, (size_t)(count * each), (fbq_stream)(uintptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

typedef fbq_status (*append_fn)(const fbq_cache *, int, int, const int32_t *, const int32_t *, const void *, int64_t, const void *, int64_t, fbq_stream);

// append(address of fbq_cache_append, address of the fbq_cache, its type, int32, layer, k, v, start, q_start, stream) -> status, or None
static PyObject *append(PyObject *self, PyObject *const *arg, Py_ssize_t n)
{
    (void)self;
    if (n != 10) {
        PyErr_SetString(PyExc_TypeError, "ten arguments");
        return NULL;
    }
    unsigned long long fn, cache, layer, stream, start, q_start, count;
    tokens_t k, v;
    if (!whole_number(arg[0], &fn) || !whole_number(arg[1], &cache) || !fn || !cache) return not_as_expected();
    const fbq_cache *const c = (const fbq_cache *)(uintptr_t)cache;
    const int ok = whole_number(arg[4], &layer) && layer <= INT32_MAX && whole_number(arg[9], &stream) && tokens(arg[5], arg[2], &k) && tokens(arg[6], arg[2], &v) && k.T == v.T &&
                   k.T <= INT32_MAX && k.heads == c->desc.kv_heads && v.heads == k.heads && k.dim == c->desc.head_dim && v.dim == k.dim &&
                   list(arg[7], arg[3], c->rows, &start, &count) && list(arg[8], arg[3], c->rows + 1LL, &q_start, &count);
    if (!ok) return not_as_expected();
    fbq_status st;
    Py_BEGIN_ALLOW_THREADS
    st = ((append_fn)(uintptr_t)fn)(c, (int)layer, (int)k.T, (const int32_t *)(uintptr_t)q_start, (const int32_t *)(uintptr_t)start, (const void *)(uintptr_t)k.at, k.stride,
                                    (const void *)(uintptr_t)v.at, v.stride, (fbq_stream)(uintptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

static PyMethodDef methods[] = {{"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, "fbq_linear of one layer; None: not as expected, nothing done"},
                                {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, "fbq_attention; None: not as expected, nothing done"},
                                {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, "fbq_cache_append; None: not as expected, nothing done"},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fbq_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fbq_call(void)
{
    static const char *const tensors[5] = {"qweight", "scales", "zeros", "At", "Bt"};
    struct { PyObject **to; const char *name; } all[] = {
        {&s_is_cuda, "is_cuda"}, {&s_is_contiguous, "is_contiguous"}, {&s_data_ptr, "data_ptr"}, {&s_numel, "numel"}, {&s_element_size, "element_size"},
        {&s_desc, "desc"}, {&s_N, "N"}, {&s_K, "K"}, {&s_r, "r"}, {&s_bits, "bits"}, {&s_group, "group"}, {&s_shape, "shape"}, {&s_dtype, "dtype"}, {&s_stride, "stride"}};
    for (size_t i = 0; i < sizeof(all) / sizeof(all[0]); ++i)
        if (!(*all[i].to = PyUnicode_InternFromString(all[i].name))) return NULL;
    for (int i = 0; i < 5; ++i)
        if (!(s_tensor[i] = PyUnicode_InternFromString(tensors[i]))) return NULL;
    return PyModule_Create(&module);
}
