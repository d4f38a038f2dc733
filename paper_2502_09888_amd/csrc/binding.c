/* The attention entry points of include/climber.h, and those on pages and positions, as Python calls, for callers whose calls are short: converts what a
 * call passes (tensors, device pointers, None; numbers; ctypes structures) in C.  By ctypes the conversions took 1.6 of a call's 4.9 us on the
 * host (4.9 -> 3.6), and two fp32 calls of one small user 10.5 us as a pass for 8.3 in their kernels, 8.7 this way.
 *
 * A function returns the entry point's code, or None where an argument is none of these: climber.py then takes ctypes' way,
 * which converts it or refuses it.  Nothing is kept from one call for the next. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/climber.h"

static __typeof__(&climber_attn_history) attn_history_fn;
static __typeof__(&climber_attn_sumi) attn_sumi_fn;
static __typeof__(&climber_attn_history_bias) attn_history_bias_fn;
static __typeof__(&climber_attn_sumi_bias) attn_sumi_bias_fn;
static __typeof__(&climber_attn_history_paged) attn_history_paged_fn;
static __typeof__(&climber_attn_sumi_paged) attn_sumi_paged_fn;
static __typeof__(&climber_paged_evict) paged_evict_fn;
static __typeof__(&climber_attn_history_paged8) attn_history_paged8_fn;
static __typeof__(&climber_attn_sumi_paged8) attn_sumi_paged8_fn;
static __typeof__(&climber_pages_fork) pages_fork_fn;
static __typeof__(&climber_pages_extend) pages_extend_fn;
static __typeof__(&climber_pages_compact) pages_compact_fn;
static __typeof__(&climber_paged_copy) paged_copy_fn;
static __typeof__(&climber_paged8_copy) paged8_copy_fn;
static __typeof__(&climber_rotary) rotary_fn;
static PyObject *pool_type, *rotary_type, *bf16_dtype, *f32_dtype, *i32_dtype, *s_dtype, *s_get_device, *s_is_contiguous;
static PyObject *config_type, *bias_type, *current_device, *raw_stream, *paged_type, *paged8_type, *s_data_ptr, *s_cuda_stream, *s_shape, *s_stride, *s_nbytes;

static int unsigned_of(PyObject *o, void **p) /* takes the reference */
{
    if (!o) return 0;
    const int ok = PyLong_Check(o);
    if (ok) *p = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(o);
    Py_DECREF(o);
    return ok && !PyErr_Occurred();
}

static int pointer(PyObject *o, void **p)
{
    if (o == Py_None) return *p = NULL, 1;
    if (PyLong_Check(o)) return unsigned_of(Py_NewRef(o), p);
    return unsigned_of(PyObject_CallMethodNoArgs(o, s_data_ptr), p);
}

/* at: the device whose current stream is meant, where the caller knows that it is the current one; None: not known */
static int stream_of(PyObject *o, PyObject *at, void **p)
{
    if (o == Py_None) { /* torch's current one */
        PyObject *dev = at == Py_None ? PyObject_CallNoArgs(current_device) : Py_NewRef(at);
        PyObject *s = dev ? PyObject_CallOneArg(raw_stream, dev) : NULL;
        Py_XDECREF(dev);
        return unsigned_of(s, p);
    }
    if (PyLong_Check(o)) return unsigned_of(Py_NewRef(o), p);
    return unsigned_of(PyObject_GetAttr(o, s_cuda_stream), p);
}

static int number(PyObject *o, int32_t *v)
{
    if (!PyLong_Check(o)) return 0;
    int over;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    *v = (int32_t)x;
    return !over && x == *v;
}

static int structure(PyObject *o, PyObject *type, size_t bytes, Py_buffer *b)
{
    if (!PyObject_TypeCheck(o, (PyTypeObject *)type)) return 0;
    if (PyObject_GetBuffer(o, b, PyBUF_SIMPLE)) return 0;
    if ((size_t)b->len == bytes) return 1;
    PyBuffer_Release(b);
    return 0;
}

static PyObject *elsewhere(void)
{
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* cfg, tau, q, k, v, scen, beh, cache, layer, o[, bias], stream */
static PyObject *history(PyObject *const *a, Py_ssize_t n, int with_bias)
{
    if (n != 11 + with_bias) return elsewhere();
    void *p[8], *o, *s;
    int32_t layer;
    Py_buffer cfg, bias;
    for (int i = 1; i < 8; ++i)
        if (!pointer(a[i], &p[i])) return elsewhere();
    if (!number(a[8], &layer) || !pointer(a[9], &o) || !stream_of(a[n - 1], Py_None, &s)) return elsewhere();
    if (!structure(a[0], config_type, sizeof(climber_config), &cfg)) return elsewhere();
    if (with_bias && !structure(a[10], bias_type, sizeof(climber_rel_bias), &bias)) return PyBuffer_Release(&cfg), elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    if (with_bias) code = attn_history_bias_fn(cfg.buf, p[1], p[2], p[3], p[4], p[5], p[6], p[7], layer, o, bias.buf, s);
    else code = attn_history_fn(cfg.buf, p[1], p[2], p[3], p[4], p[5], p[6], p[7], layer, o, s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&cfg);
    if (with_bias) PyBuffer_Release(&bias);
    return PyLong_FromLong(code);
}

/* cfg, tau, cache, layer, q, k, v, cand_off, m_total, m_max, scen, beh, o[, bias], stream */
static PyObject *sumi(PyObject *const *a, Py_ssize_t n, int with_bias)
{
    if (n != 14 + with_bias) return elsewhere();
    void *p[13], *s;
    int32_t layer, m_total, m_max;
    Py_buffer cfg, bias;
    for (int i = 1; i < 13; ++i)
        if (i != 3 && i != 8 && i != 9 && !pointer(a[i], &p[i])) return elsewhere();
    if (!number(a[3], &layer) || !number(a[8], &m_total) || !number(a[9], &m_max) || !stream_of(a[n - 1], Py_None, &s)) return elsewhere();
    if (!structure(a[0], config_type, sizeof(climber_config), &cfg)) return elsewhere();
    if (with_bias && !structure(a[13], bias_type, sizeof(climber_rel_bias), &bias)) return PyBuffer_Release(&cfg), elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    if (with_bias) code = attn_sumi_bias_fn(cfg.buf, p[1], p[2], layer, p[4], p[5], p[6], p[7], m_total, m_max, p[10], p[11], p[12], bias.buf, s);
    else code = attn_sumi_fn(cfg.buf, p[1], p[2], layer, p[4], p[5], p[6], p[7], m_total, m_max, p[10], p[11], p[12], s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&cfg);
    if (with_bias) PyBuffer_Release(&bias);
    return PyLong_FromLong(code);
}

static PyObject *attn_history(PyObject *m, PyObject *const *a, Py_ssize_t n) { return history(a, n, 0); }
static PyObject *attn_history_bias(PyObject *m, PyObject *const *a, Py_ssize_t n) { return history(a, n, 1); }
static PyObject *attn_sumi(PyObject *m, PyObject *const *a, Py_ssize_t n) { return sumi(a, n, 0); }
static PyObject *attn_sumi_bias(PyObject *m, PyObject *const *a, Py_ssize_t n) { return sumi(a, n, 1); }

/* elements from one row to the next, as climber.py's _pitch; where a type is given, of m rows or more of `least` such elements or more */
static int pitch(PyObject *o, int64_t width, PyObject *dtype, int64_t m, int64_t least, int64_t *ld)
{
    if (o == Py_None || PyLong_Check(o)) return *ld = width, 1;
    if (dtype) {
        PyObject *t = PyObject_GetAttr(o, s_dtype);
        Py_XDECREF(t);
        if (t != dtype) return 0;
    }
    PyObject *shape = PyObject_GetAttr(o, s_shape), *stride = shape ? PyObject_CallMethodNoArgs(o, s_stride) : NULL;
    int ok = stride && PyTuple_Check(shape) && PyTuple_Check(stride) && PyTuple_GET_SIZE(shape) > 0 && PyTuple_GET_SIZE(shape) == PyTuple_GET_SIZE(stride);
    if (ok) {
        int64_t inner = 1;
        for (Py_ssize_t i = PyTuple_GET_SIZE(shape) - 1; ok && i > 0; --i) {
            const int64_t n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
            ok = n == 1 || PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i)) == inner;
            inner *= n;
        }
        const int64_t rows = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0));
        *ld = rows > 1 ? PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0)) : inner > width ? inner : width;
        if (dtype) ok = ok && rows >= m && inner >= least;
    }
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    return ok && !PyErr_Occurred();
}

static int bytes_of(PyObject *o, size_t *n)
{
    void *x = NULL;
    if (o != Py_None && (PyLong_Check(o) || !unsigned_of(PyObject_GetAttr(o, s_nbytes), &x))) return 0;
    *n = (size_t)(uintptr_t)x;
    return 1;
}

/* A tensor on device `at` (a number; None: not known, then any tensor; pointers and None are taken as they are) */
static int lies_on(PyObject *o, PyObject *at)
{
    if (at == Py_None || o == Py_None || PyLong_Check(o)) return 1;
    PyObject *d = PyObject_CallMethodNoArgs(o, s_get_device);
    const int ok = d && PyObject_RichCompareBool(d, at, Py_EQ) == 1;
    Py_XDECREF(d);
    return ok;
}

/* A tensor of at least n elements of a type of 4 bytes, one behind the other (pointers and None are taken as they are) */
static int whole(PyObject *o, PyObject *dtype, int64_t n)
{
    if (o == Py_None || PyLong_Check(o)) return 1;
    PyObject *t = PyObject_GetAttr(o, s_dtype), *one = t == dtype ? PyObject_CallMethodNoArgs(o, s_is_contiguous) : NULL;
    size_t bytes;
    const int ok = one == Py_True && bytes_of(o, &bytes) && bytes / 4 >= (uint64_t)n;
    Py_XDECREF(t);
    Py_XDECREF(one);
    return ok;
}
static int ints_of(PyObject *o, int64_t n, void **p) { return whole(o, i32_dtype, n) && pointer(o, p); }

/* cfg, tau, kv, q, k, v, off, m_total, m_max, scen, beh[, stamp], o, workspace, stream[, device] */
static PyObject *paged(PyObject *const *a, Py_ssize_t n, int appends, int bits8)
{
    if (bits8) {
        if (n != 15 + appends) return elsewhere();
        --n;
        for (Py_ssize_t i = 1; i < n - 1; ++i)
            if (i != 2 && i != 7 && i != 8 && !lies_on(a[i], a[n])) return elsewhere();
    }
    if (n != 14 + appends) return elsewhere();
    void *p[14], *s;
    int32_t m_total, m_max;
    int64_t ld_q, ld_kv, ld_v, ld_o;
    size_t ws_bytes;
    Py_buffer cfg, kv;
    const Py_ssize_t o = 11 + appends;
    for (Py_ssize_t i = 1; i < n - 1; ++i)
        if (i != 2 && i != 7 && i != 8 && !pointer(a[i], &p[i])) return elsewhere();
    if (!number(a[7], &m_total) || !number(a[8], &m_max) || !bytes_of(a[o + 1], &ws_bytes) || !stream_of(a[n - 1], bits8 ? a[n] : Py_None, &s)) return elsewhere();
    if (!structure(a[0], config_type, sizeof(climber_config), &cfg)) return elsewhere();
    if (bits8 ? !paged8_type || !structure(a[2], paged8_type, sizeof(climber_paged_kv8), &kv) : !structure(a[2], paged_type, sizeof(climber_paged_kv), &kv))
        return PyBuffer_Release(&cfg), elsewhere();
    const climber_config *c = cfg.buf;
    const climber_paged_kv *cache = kv.buf; /* (a climber_paged_kv8 begins with it) */
    const int64_t wide = c->d_model, kv_wide = (int64_t)cache->n_kv_heads * c->d_head;
    int code = 0, ok = 1;
    PyObject *rows = NULL; /* their type, where it is looked at: in 8 bits, on a known device, with rows at all */
    if (bits8 && a[n] != Py_None && m_total > 0 && bf16_dtype) {
        rows = bf16_dtype;
        ok = whole(a[1], f32_dtype, (int64_t)c->n_scen * c->n_beh) && whole(a[6], i32_dtype, (int64_t)cache->n_seqs + 1);
        for (Py_ssize_t i = 9; ok && i < o; ++i) ok = whole(a[i], i32_dtype, m_total);
    }
    ok = ok && pitch(a[3], wide, rows, m_total, wide, &ld_q) && pitch(a[4], kv_wide, rows, m_total, kv_wide, &ld_kv) &&
         pitch(a[5], ld_kv, rows, m_total, kv_wide, &ld_v) && ld_v == ld_kv && pitch(a[o], wide, rows, m_total, wide, &ld_o);
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        if (bits8 && appends) code = attn_history_paged8_fn(c, p[1], kv.buf, p[3], ld_q, p[4], p[5], ld_kv, p[6], m_total, m_max, p[9], p[10], p[11], p[12], ld_o, p[13], ws_bytes, s);
        else if (bits8) code = attn_sumi_paged8_fn(c, p[1], kv.buf, p[3], ld_q, p[4], p[5], ld_kv, p[6], m_total, m_max, p[9], p[10], p[11], ld_o, p[12], ws_bytes, s);
        else if (appends) code = attn_history_paged_fn(c, p[1], kv.buf, p[3], ld_q, p[4], p[5], ld_kv, p[6], m_total, m_max, p[9], p[10], p[11], p[12], ld_o, p[13], ws_bytes, s);
        else code = attn_sumi_paged_fn(c, p[1], kv.buf, p[3], ld_q, p[4], p[5], ld_kv, p[6], m_total, m_max, p[9], p[10], p[11], ld_o, p[12], ws_bytes, s);
        Py_END_ALLOW_THREADS
    }
    PyBuffer_Release(&cfg);
    PyBuffer_Release(&kv);
    return ok ? PyLong_FromLong(code) : elsewhere();
}

static PyObject *attn_history_paged(PyObject *m, PyObject *const *a, Py_ssize_t n) { return paged(a, n, 1, 0); }
static PyObject *attn_sumi_paged(PyObject *m, PyObject *const *a, Py_ssize_t n) { return paged(a, n, 0, 0); }
static PyObject *attn_history_paged8(PyObject *m, PyObject *const *a, Py_ssize_t n) { return paged(a, n, 1, 1); }
static PyObject *attn_sumi_paged8(PyObject *m, PyObject *const *a, Py_ssize_t n) { return paged(a, n, 0, 1); }

/* cfg, kv, rank, budget, keep_from, len_out, src, workspace, stream */
static PyObject *paged_evict(PyObject *m, PyObject *const *a, Py_ssize_t n)
{
    if (n != 9) return elsewhere();
    void *p[8], *s;
    size_t ws_bytes;
    Py_buffer cfg, kv;
    for (int i = 2; i < 8; ++i)
        if (!pointer(a[i], &p[i])) return elsewhere();
    if (!bytes_of(a[7], &ws_bytes) || !stream_of(a[8], Py_None, &s)) return elsewhere();
    if (!structure(a[0], config_type, sizeof(climber_config), &cfg)) return elsewhere();
    if (!structure(a[1], paged_type, sizeof(climber_paged_kv), &kv)) return PyBuffer_Release(&cfg), elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = paged_evict_fn(cfg.buf, kv.buf, p[2], p[3], p[4], p[5], p[6], p[7], ws_bytes, s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&cfg);
    PyBuffer_Release(&kv);
    return PyLong_FromLong(code);
}

/* pool, n pointers (i: to n_seqs * seqs[i] + pages / 2 * halves[i] + more[i] integers), workspace, stream, device */
static int pool_call(PyObject *const *a, Py_ssize_t n, int pointers, const int (*sizes)[3], Py_buffer *pool, void **p, size_t *ws_bytes, void **s)
{
    if (n != pointers + 4 || !pool_type) return 0;
    for (int i = 1; i <= pointers + 1; ++i)
        if (!lies_on(a[i], a[n - 1])) return 0;
    if (!pointer(a[pointers + 1], &p[pointers + 1]) || !bytes_of(a[n - 3], ws_bytes) || !stream_of(a[n - 2], a[n - 1], s) ||
        !structure(a[0], pool_type, sizeof(climber_page_pool), pool))
        return 0;
    const climber_page_pool *c = pool->buf;
    for (int i = 1; i <= pointers; ++i) {
        const int *x = sizes[i - 1];
        if (!ints_of(a[i], (int64_t)x[0] * c->n_seqs + (int64_t)x[1] * (c->n_pages / 2) + x[2], &p[i])) return PyBuffer_Release(pool), 0;
    }
    return 1;
}
static PyObject *pages_fork(PyObject *m, PyObject *const *a, Py_ssize_t n) /* parent, keep, status */
{
    Py_buffer pool;
    void *p[5], *s;
    size_t ws;
    static const int sizes[3][3] = {{1, 0, 0}, {1, 0, 0}, {0, 0, 1}};
    if (!pool_call(a, n, 3, sizes, &pool, p, &ws, &s)) return elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = pages_fork_fn(pool.buf, p[1], p[2], p[3], p[4], ws, s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&pool);
    return PyLong_FromLong(code);
}
static PyObject *pages_extend(PyObject *m, PyObject *const *a, Py_ssize_t n) /* rows, copies, counts, status */
{
    Py_buffer pool;
    void *p[6], *s;
    size_t ws;
    static const int sizes[4][3] = {{1, 0, 0}, {3, 0, 0}, {0, 0, 2}, {0, 0, 1}};
    if (!pool_call(a, n, 4, sizes, &pool, p, &ws, &s)) return elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = pages_extend_fn(pool.buf, p[1], p[2], p[3], p[4], p[5], ws, s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&pool);
    return PyLong_FromLong(code);
}
static PyObject *pages_compact(PyObject *m, PyObject *const *a, Py_ssize_t n) /* copies, counts, status */
{
    Py_buffer pool;
    void *p[5], *s;
    size_t ws;
    static const int sizes[3][3] = {{0, 3, 0}, {0, 0, 2}, {0, 0, 1}};
    if (!pool_call(a, n, 3, sizes, &pool, p, &ws, &s)) return elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = pages_compact_fn(pool.buf, p[1], p[2], p[3], p[4], ws, s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&pool);
    return PyLong_FromLong(code);
}

/* cfg, kv, copies, counts, max_copies, stream, device */
static PyObject *copy(PyObject *const *a, Py_ssize_t n, int bits8)
{
    if (n != 7 || !paged8_type || !lies_on(a[2], a[6]) || !lies_on(a[3], a[6])) return elsewhere();
    Py_buffer cfg, kv;
    void *copies, *counts, *s;
    int32_t most;
    if (!number(a[4], &most) || !ints_of(a[2], 3 * (int64_t)(most < 0 ? 0 : most), &copies) || !ints_of(a[3], 1, &counts) || !stream_of(a[5], a[6], &s)) return elsewhere();
    if (!structure(a[0], config_type, sizeof(climber_config), &cfg)) return elsewhere();
    if (bits8 ? !structure(a[1], paged8_type, sizeof(climber_paged_kv8), &kv) : !structure(a[1], paged_type, sizeof(climber_paged_kv), &kv))
        return PyBuffer_Release(&cfg), elsewhere();
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = bits8 ? paged8_copy_fn(cfg.buf, kv.buf, copies, counts, most, s) : paged_copy_fn(cfg.buf, kv.buf, copies, counts, most, s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&cfg);
    PyBuffer_Release(&kv);
    return PyLong_FromLong(code);
}
static PyObject *paged_copy(PyObject *m, PyObject *const *a, Py_ssize_t n) { return copy(a, n, 0); }
static PyObject *paged8_copy(PyObject *m, PyObject *const *a, Py_ssize_t n) { return copy(a, n, 1); }

/* A tensor of m (or, -1, any number of) rows of `width` elements of a type, one behind the other: its pointer and pitch. */
static int rows_of(PyObject *o, int64_t width, PyObject *dtype, int64_t *m, void **p, int64_t *ld)
{
    PyObject *t = PyObject_GetAttr(o, s_dtype), *shape = t == dtype ? PyObject_GetAttr(o, s_shape) : NULL;
    PyObject *stride = shape ? PyObject_CallMethodNoArgs(o, s_stride) : NULL;
    int ok = stride && PyTuple_Check(shape) && PyTuple_Check(stride) && PyTuple_GET_SIZE(shape) > 0 && PyTuple_GET_SIZE(shape) == PyTuple_GET_SIZE(stride);
    if (ok) {
        int64_t inner = 1;
        for (Py_ssize_t i = PyTuple_GET_SIZE(shape) - 1; ok && i > 0; --i) {
            const int64_t n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
            ok = n == 1 || PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i)) == inner;
            inner *= n;
        }
        const int64_t rows = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0));
        if (*m < 0) *m = rows;
        ok = ok && rows == *m && inner == width && !PyErr_Occurred();
        *ld = rows > 1 ? PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0)) : width;
    }
    Py_XDECREF(t);
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    return ok && pointer(o, p);
}

/* cfg, plan, pos, n_kv_heads, q, k, q_out, k_out, stream, device */
static PyObject *rotary(PyObject *m, PyObject *const *a, Py_ssize_t n)
{
    if (n != 10 || !rotary_type) return elsewhere();
    for (int i = 2; i < 8; ++i)
        if (i != 3 && !lies_on(a[i], a[9])) return elsewhere();
    Py_buffer cfg, plan;
    void *pos, *p[4] = {NULL, NULL, NULL, NULL}, *s;
    int32_t n_kv;
    int64_t rows = -1, ld[4] = {0, 0, 0, 0};
    if (!number(a[3], &n_kv) || n_kv < 0 || !stream_of(a[8], a[9], &s) || !structure(a[0], config_type, sizeof(climber_config), &cfg)) return elsewhere();
    if (!structure(a[1], rotary_type, sizeof(climber_rotary_plan), &plan)) return PyBuffer_Release(&cfg), elsewhere();
    const climber_config *c = cfg.buf;
    const int64_t wide = c->d_model, kv_wide = (int64_t)n_kv * c->d_head;
    PyObject *dtype = c->dtype == CLIMBER_BF16 ? bf16_dtype : f32_dtype;
    int ok = rows_of(a[4], wide, dtype, &rows, &p[0], &ld[0]) && rows_of(a[6], wide, dtype, &rows, &p[2], &ld[2]);
    if (ok && n_kv) ok = rows_of(a[5], kv_wide, dtype, &rows, &p[1], &ld[1]) && rows_of(a[7], kv_wide, dtype, &rows, &p[3], &ld[3]);
    int64_t ld_pos = 1;
    ok = ok && rows_of(a[2], 1, i32_dtype, &rows, &pos, &ld_pos) && ld_pos == 1;
    int code = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        code = rotary_fn(c, plan.buf, pos, rows, n_kv, p[0], ld[0], p[1], ld[1], p[2], ld[2], p[3], ld[3], s);
        Py_END_ALLOW_THREADS
    }
    PyBuffer_Release(&cfg);
    PyBuffer_Release(&plan);
    return ok ? PyLong_FromLong(code) : elsewhere();
}

/* bind_pages(addresses of fork, extend, compact, the two copies and rotary, PagePool, RotaryPlan, torch.bfloat16, torch.float32, torch.int32) */
static PyObject *bind_pages(PyObject *m, PyObject *args)
{
    unsigned long long f[6];
    PyObject *t[5];
    if (!PyArg_ParseTuple(args, "KKKKKKO!O!OOO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &PyType_Type, &t[0], &PyType_Type, &t[1], &t[2], &t[3], &t[4]))
        return NULL;
    pages_fork_fn = (__typeof__(pages_fork_fn))(uintptr_t)f[0];
    pages_extend_fn = (__typeof__(pages_extend_fn))(uintptr_t)f[1];
    pages_compact_fn = (__typeof__(pages_compact_fn))(uintptr_t)f[2];
    paged_copy_fn = (__typeof__(paged_copy_fn))(uintptr_t)f[3];
    paged8_copy_fn = (__typeof__(paged8_copy_fn))(uintptr_t)f[4];
    rotary_fn = (__typeof__(rotary_fn))(uintptr_t)f[5];
    PyObject **const to[5] = {&pool_type, &rotary_type, &bf16_dtype, &f32_dtype, &i32_dtype};
    for (int i = 0; i < 5; ++i) {
        PyObject *was = *to[i];
        *to[i] = Py_NewRef(t[i]);
        Py_XDECREF(was);
    }
    Py_RETURN_NONE;
}

/* bind(addresses of the four entry points, Config, RelBias, torch.cuda.current_device, torch's raw current stream
 *      [, addresses of the three on a paged cache, PagedKV[, of the two on one in 8 bits, PagedKV8]]) */
static PyObject *bind(PyObject *m, PyObject *args)
{
    unsigned long long f[4], g[5] = {0, 0, 0, 0, 0};
    PyObject *t[6] = {NULL};
    if (!PyArg_ParseTuple(args, "KKKKO!O!OO|KKKO!KKO!", &f[0], &f[1], &f[2], &f[3], &PyType_Type, &t[0], &PyType_Type, &t[1], &t[2], &t[3], &g[0],
                          &g[1], &g[2], &PyType_Type, &t[4], &g[3], &g[4], &PyType_Type, &t[5]))
        return NULL;
    if (t[5]) {
        attn_history_paged8_fn = (__typeof__(attn_history_paged8_fn))(uintptr_t)g[3];
        attn_sumi_paged8_fn = (__typeof__(attn_sumi_paged8_fn))(uintptr_t)g[4];
    }
    if (t[4]) {
        attn_history_paged_fn = (__typeof__(attn_history_paged_fn))(uintptr_t)g[0];
        attn_sumi_paged_fn = (__typeof__(attn_sumi_paged_fn))(uintptr_t)g[1];
        paged_evict_fn = (__typeof__(paged_evict_fn))(uintptr_t)g[2];
    }
    attn_history_fn = (__typeof__(attn_history_fn))(uintptr_t)f[0];
    attn_sumi_fn = (__typeof__(attn_sumi_fn))(uintptr_t)f[1];
    attn_history_bias_fn = (__typeof__(attn_history_bias_fn))(uintptr_t)f[2];
    attn_sumi_bias_fn = (__typeof__(attn_sumi_bias_fn))(uintptr_t)f[3];
    PyObject **const to[6] = {&config_type, &bias_type, &current_device, &raw_stream, &paged_type, &paged8_type};
    for (int i = 0; i < 6 && t[i]; ++i) {
        PyObject *was = *to[i];
        *to[i] = Py_NewRef(t[i]);
        Py_XDECREF(was);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, NULL},
    {"attn_history", (PyCFunction)(void (*)(void))attn_history, METH_FASTCALL, NULL},
    {"attn_history_bias", (PyCFunction)(void (*)(void))attn_history_bias, METH_FASTCALL, NULL},
    {"attn_sumi", (PyCFunction)(void (*)(void))attn_sumi, METH_FASTCALL, NULL},
    {"attn_sumi_bias", (PyCFunction)(void (*)(void))attn_sumi_bias, METH_FASTCALL, NULL},
    {"attn_history_paged", (PyCFunction)(void (*)(void))attn_history_paged, METH_FASTCALL, NULL},
    {"attn_sumi_paged", (PyCFunction)(void (*)(void))attn_sumi_paged, METH_FASTCALL, NULL},
    {"attn_history_paged8", (PyCFunction)(void (*)(void))attn_history_paged8, METH_FASTCALL, NULL},
    {"attn_sumi_paged8", (PyCFunction)(void (*)(void))attn_sumi_paged8, METH_FASTCALL, NULL},
    {"bind_pages", bind_pages, METH_VARARGS, NULL},
    {"pages_fork", (PyCFunction)(void (*)(void))pages_fork, METH_FASTCALL, NULL},
    {"pages_extend", (PyCFunction)(void (*)(void))pages_extend, METH_FASTCALL, NULL},
    {"pages_compact", (PyCFunction)(void (*)(void))pages_compact, METH_FASTCALL, NULL},
    {"paged_copy", (PyCFunction)(void (*)(void))paged_copy, METH_FASTCALL, NULL},
    {"paged8_copy", (PyCFunction)(void (*)(void))paged8_copy, METH_FASTCALL, NULL},
    {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, NULL},
    {"paged_evict", (PyCFunction)(void (*)(void))paged_evict, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__native(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    return s_is_contiguous && s_dtype && s_get_device && s_data_ptr && s_cuda_stream && s_shape && s_stride && s_nbytes ? PyModule_Create(&module) : NULL;
}
