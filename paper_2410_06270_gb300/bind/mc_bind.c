/*
 * mc_bind.c -- argument marshalling of the calls that a decode step makes many times a
 * second (kv_append, attn_decode, attn_prefill, their 4-bit forms, kv4_read, kv_plan, residual_norm), as a CPython extension: what the binding
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

static append_fn c_append[2]; /* to the 16-bit cache, to the 4-bit one */
static attn_fn c_attn[4];     /* decode, prefill; over the 4-bit cache */
typedef int (*read_fn)(const mc_kv_cache *, const mc_kv_batch *, void *, void *, void *, void *);
typedef int (*plan_fn)(const mc_kv_pool *, const int32_t *, const int32_t *, const uint8_t *, int, int, int32_t *, int, int32_t *, int32_t *,
                       int32_t *, int64_t *, int64_t *, void *, size_t, void *);
typedef int (*residual_fn)(const mc_residual_norm_args *, void *);
static read_fn c_read;
static plan_fn c_plan;
static residual_fn c_residual;
static PyObject *t_empty, *t_stream, *t_device, *t_float32, *t_int32, *t_uint8, *t_int64, *t_bf16, *t_fp16;
static PyObject *n_state, *n_shape, *n_stride, *n_dtype, *n_device, *n_get_device, *n_data_ptr, *n_is_contiguous, *n_ref, *n_index,
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

/* append(bits4, cache, batch, q, k, v, rope, interleaved, q_norm, k_norm, eps, q_out, workspace) */
static PyObject *append(PyObject *self, PyObject *const *a, Py_ssize_t na)
{
    (void)self;
    Call c = {0};
    const int bits4 = na == 13 ? PyObject_IsTrue(*a++) : -1;
    if (bits4 < 0 || !begin(&c, a[0], a[1])) return leave(&c);
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
    rc = c_append[bits4](c.cache, c.batch, q, qs, k, ks, v, vs, heads, qn, kn, (float)eps, (const float *)rope, (int)rope_n[0], (int)rope_n[1],
                  inter, o, (void *)ws, (void *)(intptr_t)st);
    Py_END_ALLOW_THREADS
    end(&c);
    if (rc) {
        Py_DECREF(out);
        return PyLong_FromLong(rc);
    }
    return out;
}

/* attention(which, cache, batch, q, scale, softcap, window, slopes, prefix, out, with_lse, workspace) */
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
    const long kind = PyLong_AsLong(a[0]);
    const int with_lse = PyObject_IsTrue(a[10]);
    const int64_t st = stream_of(&c);
    if (st < 0 || kind < 0 || kind > 3 || with_lse < 0 || window != o.window || PyErr_Occurred()) return leave(&c);
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

/* kv4_read(cache, batch, k, v, workspace) */
static PyObject *kv4_read(PyObject *self, PyObject *const *a, Py_ssize_t na)
{
    (void)self;
    Call c = {0};
    if (na != 5 || !begin(&c, a[0], a[1]) || c.batch->tokens < 1) return leave(&c);
    int64_t n[1];
    const void *ws = NULL;
    if (!side(&c, a[4], t_uint8, 1, n, &ws) || (a[4] != Py_None && n[0] < 256)) return leave(&c);
    const int64_t st = stream_of(&c);
    if (st < 0 || PyErr_Occurred()) return leave(&c);
    PyObject *out[2] = {NULL, NULL};
    for (int i = 0; i < 2; ++i) {
        int got;
        int64_t os;
        if (a[2 + i] == Py_None) {
            out[i] = empty3(&c, c.batch->tokens, c.cache->kv_heads, c.cache->head_dim, c.dtype);
        } else if (rows(&c, a[2 + i], c.cache->kv_heads, &got, &os) && is_true(a[2 + i], n_is_contiguous)) {
            out[i] = a[2 + i];
            Py_INCREF(out[i]);
        }
        if (!out[i]) {
            Py_XDECREF(out[0]);
            return leave(&c);
        }
    }
    void *k = ptr_of(out[0]), *v = ptr_of(out[1]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c_read(c.cache, c.batch, k, v, (void *)ws, (void *)(intptr_t)st);
    Py_END_ALLOW_THREADS
    end(&c);
    PyObject *both = rc ? PyLong_FromLong(rc) : PyTuple_Pack(2, out[0], out[1]);
    Py_DECREF(out[0]);
    Py_DECREF(out[1]);
    return both;
}

/* Sizes and strides of a tensor of `dims` dimensions and this type on device `index`; 0: not a plain case. */
static int tensor(PyObject *t, PyObject *dtype, int64_t index, int dims, int64_t *n, int64_t *s)
{
    int ok = 0;
    PyObject *sh = PyObject_GetAttr(t, n_shape), *st = NULL, *dt = NULL;
    if (sh && PyTuple_Check(sh) && PyTuple_GET_SIZE(sh) == dims && (st = PyObject_CallMethodNoArgs(t, n_stride)) && PyTuple_Check(st) &&
        (dt = PyObject_GetAttr(t, n_dtype)) && dt == dtype) {
        for (int i = 0; i < dims; ++i) {
            n[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, i));
            s[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(st, i));
        }
        ok = int_of(t, n_get_device) == index;
    }
    Py_XDECREF(sh);
    Py_XDECREF(st);
    Py_XDECREF(dt);
    return ok && !PyErr_Occurred();
}

/* n contiguous elements */
static int vec(PyObject *t, PyObject *dtype, int64_t index, int64_t n)
{
    int64_t got, s;
    return tensor(t, dtype, index, 1, &got, &s) && got == n && (s == 1 || n < 2);
}

/* a new tensor of one or two (b > 0) dimensions */
static PyObject *empty(int64_t a, int64_t b, PyObject *dtype, PyObject *device)
{
    PyObject *shape = b > 0 ? Py_BuildValue("(LL)", (long long)a, (long long)b) : Py_BuildValue("(L)", (long long)a);
    if (!shape) return NULL;
    PyObject *args[3] = {shape, dtype, device};
    PyObject *r = PyObject_Vectorcall(t_empty, args, 1, kw_empty);
    Py_DECREF(shape);
    return r;
}

/* torch's current stream if device `index` is the current one; -1 otherwise (stream_of) */
static int64_t stream_on(int64_t index)
{
    Call c = {0};
    c.index = index;
    return index < 0 ? -1 : stream_of(&c);
}

static PyObject *not_plain(PyObject **owned, int count)
{
    for (int i = 0; i < count; ++i) Py_XDECREF(owned[i]);
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* plan(pool, table, lens, add, done, tokens, lens_out, positions, slots, commit, workspace):
 * (lens_out, cu_q, positions, slots, state, tokens) */
static PyObject *plan(PyObject *self, PyObject *const *a, Py_ssize_t na)
{
    (void)self;
    enum { kLens, kCu, kPos, kSlots, kState, kDevice, kOwned };
    PyObject *o[kOwned] = {0};
    if (na != 11 || a[10] == Py_None) return not_plain(o, kOwned);
    const mc_kv_pool *pool = (const mc_kv_pool *)(uintptr_t)attr_int(a[0], n_ref);
    const int64_t index = attr_int(a[0], n_index);
    int64_t n[2], s[2], wn, wst;
    if (PyErr_Occurred() || !tensor(a[1], t_int32, index, 2, n, s)) return not_plain(o, kOwned);
    const int64_t seqs = n[0], width = n[1];
    if (seqs < 1 || seqs > 0x7fffffff || width < 1 || width > 0x7fffffff || (s[1] != 1 && width > 1) || (s[0] != width && seqs > 1)) return not_plain(o, kOwned);
    if (!vec(a[2], t_int32, index, seqs) || !vec(a[3], t_int32, index, seqs)) return not_plain(o, kOwned);
    if (a[4] != Py_None && !vec(a[4], t_uint8, index, seqs)) return not_plain(o, kOwned);
    if (a[6] != Py_None && !vec(a[6], t_int32, index, seqs)) return not_plain(o, kOwned);
    if (!tensor(a[10], t_uint8, index, 1, &wn, &wst) || wst != 1 || wn < 256) return not_plain(o, kOwned);
    const int64_t tokens = a[5] == Py_None ? seqs : PyLong_AsLongLong(a[5]);
    const int positions = PyObject_IsTrue(a[7]), slots = PyObject_IsTrue(a[8]), commit = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred() || tokens < 0 || tokens > 0x7fffffff) return not_plain(o, kOwned);
    const int64_t st = stream_on(index);
    if (st < 0) return not_plain(o, kOwned);
    o[kDevice] = PyObject_GetAttr(a[0], n_device);
    if (!o[kDevice]) return not_plain(o, kOwned);
    if (a[6] != Py_None) {
        o[kLens] = a[6];
        Py_INCREF(a[6]);
    } else {
        o[kLens] = empty(seqs, 0, t_int32, o[kDevice]);
    }
    o[kCu] = empty(seqs + 1, 0, t_int32, o[kDevice]);
    if (positions) o[kPos] = empty(tokens, 0, t_int32, o[kDevice]);
    else o[kPos] = Py_None, Py_INCREF(Py_None);
    if (slots) o[kSlots] = empty(tokens, 0, t_int64, o[kDevice]);
    else o[kSlots] = Py_None, Py_INCREF(Py_None);
    o[kState] = commit ? PyObject_GetAttr(a[0], n_state) : empty(2, 0, t_int64, o[kDevice]);
    for (int i = 0; i < kOwned; ++i)
        if (!o[i]) return not_plain(o, kOwned);
    const void *table = ptr_of(a[1]), *lens = ptr_of(a[2]), *add = ptr_of(a[3]), *done = a[4] == Py_None ? NULL : ptr_of(a[4]), *ws = ptr_of(a[10]);
    void *lo = ptr_of(o[kLens]), *cu = ptr_of(o[kCu]), *po = positions ? ptr_of(o[kPos]) : NULL, *sl = slots ? ptr_of(o[kSlots]) : NULL,
         *so = ptr_of(o[kState]);
    if (PyErr_Occurred()) return not_plain(o, kOwned);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c_plan(pool, lens, add, done, (int)seqs, (int)tokens, (int32_t *)table, (int)width, lo, cu, po, sl, so, (void *)ws, (size_t)wn,
                (void *)(intptr_t)st);
    Py_END_ALLOW_THREADS
    PyObject *r = rc ? PyLong_FromLong(rc) : Py_BuildValue("(OOOOOL)", o[kLens], o[kCu], o[kPos], o[kSlots], o[kState], (long long)tokens);
    for (int i = 0; i < kOwned; ++i) Py_DECREF(o[i]);
    return r;
}

/* residual(y, h, pre_norm, post_norm, gate, scale, residual_scale, eps, h_out, x): (h_out, x) */
static PyObject *residual(PyObject *self, PyObject *const *a, Py_ssize_t na)
{
    (void)self;
    enum { kType, kDevice, kHOut, kX, kOwned };
    PyObject *o[kOwned] = {0};
    if (na != 10) return not_plain(o, kOwned);
    mc_residual_norm_args r = {0};
    int64_t n[2], s[2], gn[2], gs[2], hs[2];
    o[kType] = PyObject_GetAttr(a[0], n_dtype);
    if (!o[kType] || (o[kType] != t_bf16 && o[kType] != t_fp16)) return not_plain(o, kOwned);
    const int64_t index = int_of(a[0], n_get_device);
    if (!tensor(a[0], o[kType], index, 2, n, s) || n[0] < 1 || n[0] > 0x7fffffff || n[1] < 1 || n[1] > 65536) return not_plain(o, kOwned);
    const int64_t T = n[0], H = n[1];
    /* rows of [T, H]: their stride, or 0 */
#define ROWS(t, stride) \
    (tensor(t, o[kType], index, 2, gn, gs) && gn[0] == T && gn[1] == H && (gs[1] == 1 || H == 1) && ((stride) = T > 1 ? gs[0] : H, 1))
    if (s[1] != 1 && H > 1) return not_plain(o, kOwned);
    r.y_stride = T > 1 ? s[0] : H;
    if (!ROWS(a[1], hs[0])) return not_plain(o, kOwned);
    r.h_stride = hs[0];
    for (int i = 2; i < 4; ++i)
        if (a[i] != Py_None && !vec(a[i], o[kType], index, H)) return not_plain(o, kOwned);
    if (a[4] != Py_None) {
        if (!tensor(a[4], o[kType], index, 2, gn, gs) || (gn[0] != 1 && gn[0] != T) || (gn[1] != 1 && gn[1] != H)) return not_plain(o, kOwned);
        r.gate_row = gn[0] > 1 ? gs[0] : 0;
        r.gate_col = gn[1] > 1 ? (int32_t)gs[1] : 0;
        if (gn[1] > 1 && gs[1] != 1) return not_plain(o, kOwned);
        r.gate = ptr_of(a[4]);
    }
    r.scale = (float)PyFloat_AsDouble(a[5]);
    r.residual_scale = (float)PyFloat_AsDouble(a[6]);
    r.eps = (float)PyFloat_AsDouble(a[7]);
    const int64_t st = stream_on(index);
    if (st < 0 || PyErr_Occurred()) return not_plain(o, kOwned);
    r.h_out_stride = r.x_stride = H;
    if ((a[8] == Py_None || a[9] == Py_None) && !(o[kDevice] = PyObject_GetAttr(a[0], n_device))) return not_plain(o, kOwned);
    if (a[8] == Py_None) {
        o[kHOut] = empty(T, H, o[kType], o[kDevice]);
    } else {
        if (!ROWS(a[8], r.h_out_stride)) return not_plain(o, kOwned);
        o[kHOut] = a[8];
        Py_INCREF(a[8]);
    }
    if (a[2] == Py_None) {
        o[kX] = Py_None;
        Py_INCREF(Py_None);
    } else if (a[9] == Py_None) {
        o[kX] = empty(T, H, o[kType], o[kDevice]);
    } else {
        if (!ROWS(a[9], r.x_stride)) return not_plain(o, kOwned);
        o[kX] = a[9];
        Py_INCREF(a[9]);
    }
#undef ROWS
    if (!o[kHOut] || !o[kX]) return not_plain(o, kOwned);
    r.T = (int32_t)T;
    r.H = (int32_t)H;
    r.dtype = o[kType] == t_bf16 ? MC_BF16 : MC_FP16;
    r.y = ptr_of(a[0]);
    r.h = ptr_of(a[1]);
    r.pre_norm = a[2] == Py_None ? NULL : ptr_of(a[2]);
    r.post_norm = a[3] == Py_None ? NULL : ptr_of(a[3]);
    r.h_out = ptr_of(o[kHOut]);
    r.x = o[kX] == Py_None ? NULL : ptr_of(o[kX]);
    if (PyErr_Occurred()) return not_plain(o, kOwned);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c_residual(&r, (void *)(intptr_t)st);
    Py_END_ALLOW_THREADS
    PyObject *both = rc ? PyLong_FromLong(rc) : PyTuple_Pack(2, o[kHOut], o[kX]);
    for (int i = 0; i < kOwned; ++i) Py_XDECREF(o[i]);
    return both;
}

/* setup(append, decode, prefill, append4, decode4, prefill4, read, plan, residual, empty, raw_stream, current_device, float32, int32, uint8, int64, bfloat16,
 * float16) */
static PyObject *setup(PyObject *self, PyObject *args)
{
    (void)self;
    unsigned long long f[9];
    PyObject *o[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKOOOOOOOOO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8], &o[0], &o[1], &o[2], &o[3],
                          &o[4], &o[5], &o[6], &o[7], &o[8]))
        return NULL;
    for (int i = 0; i < 2; ++i) {
        c_append[i] = (append_fn)(uintptr_t)f[3 * i];
        c_attn[2 * i] = (attn_fn)(uintptr_t)f[3 * i + 1];
        c_attn[2 * i + 1] = (attn_fn)(uintptr_t)f[3 * i + 2];
    }
    c_read = (read_fn)(uintptr_t)f[6];
    c_plan = (plan_fn)(uintptr_t)f[7];
    c_residual = (residual_fn)(uintptr_t)f[8];
    PyObject **to[9] = {&t_empty, &t_stream, &t_device, &t_float32, &t_int32, &t_uint8, &t_int64, &t_bf16, &t_fp16};
    for (int i = 0; i < 9; ++i) {
        Py_INCREF(o[i]);
        Py_XSETREF(*to[i], o[i]);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, "entry points and torch's parts"},
                                {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, ""},
                                {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, ""},
                                {"kv4_read", (PyCFunction)(void (*)(void))kv4_read, METH_FASTCALL, ""},
                                {"plan", (PyCFunction)(void (*)(void))plan, METH_FASTCALL, ""},
                                {"residual", (PyCFunction)(void (*)(void))residual, METH_FASTCALL, ""},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mcbind", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__mcbind(void)
{
    struct {
        PyObject **to;
        const char *name;
    } names[] = {{&n_shape, "shape"}, {&n_stride, "stride"}, {&n_dtype, "dtype"}, {&n_device, "device"}, {&n_get_device, "get_device"},
                 {&n_data_ptr, "data_ptr"}, {&n_is_contiguous, "is_contiguous"}, {&n_ref, "_ref"}, {&n_index, "index"}, {&n_state, "state"}};
    for (size_t i = 0; i < sizeof names / sizeof names[0]; ++i)
        if (!(*names[i].to = PyUnicode_InternFromString(names[i].name))) return NULL;
    if (!(kw_empty = Py_BuildValue("(ss)", "dtype", "device"))) return NULL;
    return PyModule_Create(&module);
}
