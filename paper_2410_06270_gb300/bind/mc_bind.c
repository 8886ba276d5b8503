/*
 * mc_bind.c -- argument marshalling of the calls that a decode step makes many times a
 * second (kv_append, attn_decode, attn_prefill), as a CPython extension: what the binding
 * does in Python with ctypes costs 6 to 8 us a call, several times such a call's kernels.
 *
 * It takes the plain cases only.  Whatever is not as it should be (a shape, a stride, a type,
 * a device, a missing workspace) is answered with None, and the Python marshalling, which
 * takes every case, says what is wrong or does the call.  An integer is the C entry point's
 * error code.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "mc.h"

typedef int (*append_fn)(const mc_kv_cache *, const mc_kv_batch *, const void *, int64_t, const void *, int64_t, const void *,
                         int64_t, int, const void *, const void *, float, const float *, int, int, int, void *, void *, void *);
typedef int (*attn_fn)(const mc_kv_cache *, const mc_kv_batch *, const void *, int64_t, int, const mc_attn_opts *, void *, int64_t,
                       float *, void *, size_t, void *);

static append_fn c_append;
static attn_fn c_attn[2]; /* decode, prefill */
static PyObject *t_empty, *t_stream, *t_device, *t_float32, *t_int32, *t_uint8;
static PyObject *n_shape, *n_stride, *n_dtype, *n_device, *n_get_device, *n_data_ptr, *n_is_contiguous, *n_ref, *n_index,
    *kw_empty;

/* a call without arguments, as an integer; -1 and an error set on failure */
static int64_t int_of(PyObject *o, PyObject *method)
{
    PyObject *r = PyObject_CallMethodNoArgs(o, method);
    if (!r) return -1;
    const int64_t v = PyLong_AsLongLong(r);
    Py_DECREF(r);
    return v;
}

static void *ptr_of(PyObject *t)
{
    PyObject *r = PyObject_CallMethodNoArgs(t, n_data_ptr);
    if (!r) return NULL;
    void *p = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(r);
    Py_DECREF(r);
    return p;
}

static int64_t attr_int(PyObject *o, PyObject *name)
{
    PyObject *r = PyObject_GetAttr(o, name);
    if (!r) return -1;
    const int64_t v = PyLong_AsLongLong(r);
    Py_DECREF(r);
    return v;
}

typedef struct {
    const mc_kv_cache *cache;
    const mc_kv_batch *batch;
    PyObject *dtype, *device; /* the cache's (owned) */
    int64_t index;
} Call;

/* 1: ready; 0: not a plain case (or an error is set) */
static int begin(Call *c, PyObject *cache, PyObject *batch)
{
    c->cache = (const mc_kv_cache *)(uintptr_t)attr_int(cache, n_ref);
    c->batch = (const mc_kv_batch *)(uintptr_t)attr_int(batch, n_ref);
    c->index = attr_int(cache, n_index);
    const int64_t other = attr_int(batch, n_index);
    c->dtype = PyObject_GetAttr(cache, n_dtype);
    c->device = PyObject_GetAttr(cache, n_device);
    return !PyErr_Occurred() && c->dtype && c->device && c->index >= 0 && other == c->index;
}

static void end(Call *c)
{
    Py_XDECREF(c->dtype);
    Py_XDECREF(c->device);
}

/* Heads and token stride of t [tokens, heads, head_dim]; 0: not a plain case. */
static int rows(const Call *c, PyObject *t, int heads, int *got, int64_t *stride)
{
    int ok = 0;
    PyObject *sh = PyObject_GetAttr(t, n_shape), *st = NULL, *dt = NULL;
    if (sh && PyTuple_Check(sh) && PyTuple_GET_SIZE(sh) == 3 && (st = PyObject_CallMethodNoArgs(t, n_stride)) && PyTuple_Check(st) &&
        PyTuple_GET_SIZE(st) == 3 && (dt = PyObject_GetAttr(t, n_dtype))) {
        int64_t n[3], s[3];
        for (int i = 0; i < 3; ++i) {
            n[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, i));
            s[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(st, i));
        }
        const int64_t D = c->cache->head_dim;
        ok = n[0] == c->batch->tokens && n[0] > 0 && n[1] > 0 && n[1] <= 4096 && (!heads || n[1] == heads) && n[2] == D && s[2] == 1 &&
             (s[1] == D || n[1] == 1) && dt == c->dtype && int_of(t, n_get_device) == c->index;
        if (n[0] == 1 && s[0] < n[1] * D) s[0] = n[1] * D; /* (a single row's stride means nothing) */
        *got = (int)n[1];
        *stride = s[0];
    }
    Py_XDECREF(sh);
    Py_XDECREF(st);
    Py_XDECREF(dt);
    return ok && !PyErr_Occurred();
}

static int is_true(PyObject *o, PyObject *method)
{
    PyObject *r = PyObject_CallMethodNoArgs(o, method);
    const int v = r == Py_True;
    Py_XDECREF(r);
    return v;
}

/* A contiguous side input of `dims` dimensions, its sizes in n; None: *p stays NULL. */
static int side(const Call *c, PyObject *t, PyObject *dtype, int dims, int64_t *n, const void **p)
{
    *p = NULL;
    if (t == Py_None) return 1;
    int ok = 0;
    PyObject *sh = PyObject_GetAttr(t, n_shape), *dt = sh ? PyObject_GetAttr(t, n_dtype) : NULL;
    if (dt && PyTuple_Check(sh) && PyTuple_GET_SIZE(sh) == dims) {
        for (int i = 0; i < dims; ++i) n[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, i));
        ok = dt == dtype && int_of(t, n_get_device) == c->index && is_true(t, n_is_contiguous);
        if (ok) *p = ptr_of(t);
    }
    Py_XDECREF(sh);
    Py_XDECREF(dt);
    return ok && !PyErr_Occurred();
}

static PyObject *empty3(const Call *c, int64_t a, int64_t b, int64_t d, PyObject *dtype)
{
    PyObject *shape = d ? Py_BuildValue("(LLL)", (long long)a, (long long)b, (long long)d) : Py_BuildValue("(LL)", (long long)a, (long long)b);
    if (!shape) return NULL;
    PyObject *args[3] = {shape, dtype, c->device};
    PyObject *r = PyObject_Vectorcall(t_empty, args, 1, kw_empty);
    Py_DECREF(shape);
    return r;
}

/* torch's current stream, if the cache's device is the current one; -1 otherwise */
static int64_t stream_of(const Call *c)
{
    PyObject *dev = PyObject_CallNoArgs(t_device);
    if (!dev) return -1;
    const int64_t d = PyLong_AsLongLong(dev);
    PyObject *s = d == c->index ? PyObject_CallOneArg(t_stream, dev) : NULL;
    Py_DECREF(dev);
    if (!s) return -1;
    const int64_t v = PyLong_AsLongLong(s);
    Py_DECREF(s);
    return v;
}

/* nothing plain: None, and no error left behind (the Python marshalling finds it again) */
static PyObject *leave(Call *c)
{
    end(c);
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* kv_append(cache, batch, q, k, v, rope, interleaved, q_norm, k_norm, eps, q_out, workspace) */
static PyObject *kv_append(PyObject *self, PyObject *const *a, Py_ssize_t na)
{
    (void)self;
    Call c = {0};
    if (na != 12 || !begin(&c, a[0], a[1])) return leave(&c);
    int heads = 0, kh;
    int64_t qs, ks, vs, os, n[2], rope_n[2] = {0, 0};
    const void *rope, *qn, *kn, *ws = NULL;
    const int D = c.cache->head_dim, kv = c.cache->kv_heads;
    if (!rows(&c, a[2], 0, &heads, &qs) || !rows(&c, a[3], kv, &kh, &ks) || !rows(&c, a[4], kv, &kh, &vs)) return leave(&c);
    if (!side(&c, a[5], t_float32, 2, rope_n, &rope)) return leave(&c);
    if (!side(&c, a[7], c.dtype, 1, n, &qn) || (qn && n[0] != D)) return leave(&c);
    if (!side(&c, a[8], c.dtype, 1, n, &kn) || (kn && n[0] != D)) return leave(&c);
    if (!side(&c, a[11], t_uint8, 1, n, &ws) || (a[11] != Py_None && n[0] < 256)) return leave(&c);
    const double eps = PyFloat_AsDouble(a[9]);
    const int inter = PyObject_IsTrue(a[6]);
    const int64_t st = stream_of(&c);
    if (st < 0 || inter < 0 || rope_n[0] > 0x7fffffff || rope_n[1] > 4096 || PyErr_Occurred()) return leave(&c);
    PyObject *out = a[10];
    if (out == Py_None) {
        out = empty3(&c, c.batch->tokens, heads, D, c.dtype);
        if (!out) return leave(&c);
    } else if (rows(&c, out, heads, &kh, &os) && is_true(out, n_is_contiguous)) {
        Py_INCREF(out);
    } else {
        return leave(&c);
    }
    const void *q = ptr_of(a[2]), *k = ptr_of(a[3]), *v = ptr_of(a[4]);
    void *o = ptr_of(out);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c_append(c.cache, c.batch, q, qs, k, ks, v, vs, heads, qn, kn, (float)eps, (const float *)rope, (int)rope_n[0], (int)rope_n[1],
                  inter, o, (void *)ws, (void *)(intptr_t)st);
    Py_END_ALLOW_THREADS
    end(&c);
    if (rc) {
        Py_DECREF(out);
        return PyLong_FromLong(rc);
    }
    return out;
}

/* attention(prefill, cache, batch, q, scale, softcap, window, slopes, prefix, out, with_lse, workspace) */
static PyObject *attention(PyObject *self, PyObject *const *a, Py_ssize_t na)
{
    (void)self;
    Call c = {0};
    if (na != 12 || !begin(&c, a[1], a[2])) return leave(&c);
    int heads = 0, got;
    int64_t qs, os, n[2], ws_n[1];
    const void *slopes, *prefix, *ws;
    if (!rows(&c, a[3], 0, &heads, &qs)) return leave(&c);
    if (!side(&c, a[7], t_float32, 1, n, &slopes) || (slopes && n[0] != heads)) return leave(&c);
    if (!side(&c, a[8], t_int32, 1, n, &prefix) || (prefix && n[0] != c.batch->seqs)) return leave(&c);
    if (a[11] == Py_None || !side(&c, a[11], t_uint8, 1, ws_n, &ws)) return leave(&c);
    mc_attn_opts o;
    o.scale = a[4] == Py_None ? (c.cache->head_dim == 64 ? 0.125f : 0.08838834764831845f) : (float)PyFloat_AsDouble(a[4]);
    o.softcap = (float)PyFloat_AsDouble(a[5]);
    const long long window = PyLong_AsLongLong(a[6]);
    o.window = (int32_t)window;
    o.slopes = (const float *)slopes;
    o.prefix = (const int32_t *)prefix;
    const int kind = PyObject_IsTrue(a[0]), with_lse = PyObject_IsTrue(a[10]);
    const int64_t st = stream_of(&c);
    if (st < 0 || kind < 0 || with_lse < 0 || window != o.window || PyErr_Occurred()) return leave(&c);
    PyObject *out = a[9], *lse = NULL;
    if (out == Py_None) {
        out = empty3(&c, c.batch->tokens, heads, c.cache->head_dim, c.dtype);
        if (!out) return leave(&c);
        os = (int64_t)heads * c.cache->head_dim;
    } else if (rows(&c, out, heads, &got, &os)) {
        Py_INCREF(out);
    } else {
        return leave(&c);
    }
    if (with_lse && !(lse = empty3(&c, c.batch->tokens, heads, 0, t_float32))) {
        Py_DECREF(out);
        return leave(&c);
    }
    const void *q = ptr_of(a[3]);
    void *po = ptr_of(out);
    float *pl = lse ? (float *)ptr_of(lse) : NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c_attn[kind](c.cache, c.batch, q, qs, heads, &o, po, os, pl, (void *)ws, (size_t)ws_n[0], (void *)(intptr_t)st);
    Py_END_ALLOW_THREADS
    end(&c);
    if (rc) {
        Py_DECREF(out);
        Py_XDECREF(lse);
        return PyLong_FromLong(rc);
    }
    if (!with_lse) return out;
    PyObject *both = PyTuple_Pack(2, out, lse);
    Py_DECREF(out);
    Py_DECREF(lse);
    return both;
}

/* setup(append, decode, prefill, empty, raw_stream, current_device, float32, int32, uint8) */
static PyObject *setup(PyObject *self, PyObject *args)
{
    (void)self;
    unsigned long long fa, fd, fp;
    PyObject *o[6];
    if (!PyArg_ParseTuple(args, "KKKOOOOOO", &fa, &fd, &fp, &o[0], &o[1], &o[2], &o[3], &o[4], &o[5])) return NULL;
    c_append = (append_fn)(uintptr_t)fa;
    c_attn[0] = (attn_fn)(uintptr_t)fd;
    c_attn[1] = (attn_fn)(uintptr_t)fp;
    PyObject **to[6] = {&t_empty, &t_stream, &t_device, &t_float32, &t_int32, &t_uint8};
    for (int i = 0; i < 6; ++i) {
        Py_INCREF(o[i]);
        Py_XSETREF(*to[i], o[i]);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, "entry points and torch's parts"},
                                {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, ""},
                                {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, ""},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mcbind", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__mcbind(void)
{
    struct {
        PyObject **to;
        const char *name;
    } names[] = {{&n_shape, "shape"}, {&n_stride, "stride"}, {&n_dtype, "dtype"}, {&n_device, "device"}, {&n_get_device, "get_device"},
                 {&n_data_ptr, "data_ptr"}, {&n_is_contiguous, "is_contiguous"}, {&n_ref, "_ref"}, {&n_index, "index"}};
    for (size_t i = 0; i < sizeof names / sizeof names[0]; ++i)
        if (!(*names[i].to = PyUnicode_InternFromString(names[i].name))) return NULL;
    if (!(kw_empty = Py_BuildValue("(ss)", "dtype", "device"))) return NULL;
    return PyModule_Create(&module);
}
