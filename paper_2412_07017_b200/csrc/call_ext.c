/* Argument marshalling of the calls that a serving step makes for every layer, as a CPython extension: the C ABI of
 * include/asynclm.h called with the addresses of tensors and arrays.  binding.py uses it where it has been built and the
 * arguments are of the ordinary kinds; everything else goes through ctypes there.
 *
 * Why: a step of few sequences is bound by the host.  Through ctypes, planning 4 sequences took 20.8 us (4.0 of them to turn the
 * four arrays into addresses) and a layer's call 4.2-4.4; so 13.8 (with the headers that such a plan no longer uploads) and
 * 3.6, of which the launch is 2.6.  A step of 4 sequences in one layer: 48.3 -> 29.0 us. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "asynclm.h"

static int (*fn_plan)(const asynclm_shape*, const asynclm_plan_options*, const asynclm_batch*, void*, size_t, void*, size_t, void*,
                      asynclm_plan_t**);
static int (*fn_append)(const asynclm_plan_t*, const void*, const void*, void*, void*);
static int (*fn_append_rope)(const asynclm_plan_t*, const void*, const void*, void*, void*, double, void*);
static int (*fn_attn)(const asynclm_plan_t*, const void*, const void*, void*, float*, void*);
static int (*fn_step)(const asynclm_plan_t*, const void*, const void*, const void*, void*, void*, float*, void*);
static int (*fn_kv8_append)(const asynclm_plan_t*, const asynclm_kv8_rows*, void*, void*, const asynclm_rope_table*, void*);
static int (*fn_kv8_attn)(const asynclm_plan_t*, const void*, const void*, const void*, void*, float*, void*);
static int (*fn_kv8_gather)(const asynclm_plan_t*, const int64_t*, const int32_t*, int64_t, const void*, const void*, void*, void*, void*);
static int (*fn_plan_shape)(const asynclm_plan_t*, asynclm_shape*, int32_t*, int32_t*);
static int (*fn_rope)(const asynclm_rope_table*, const int32_t*, int32_t, int32_t, const asynclm_rope_rows*, int32_t, void*);
static int (*fn_bounds)(const asynclm_plan_t*, const void*, void*, int32_t, void*);
static int (*fn_kv8_bounds)(const asynclm_plan_t*, const void*, const void*, void*, int32_t, void*);
static int (*fn_select)(const asynclm_plan_t*, const void*, const void*, int32_t*, void*);
static int (*fn_plan_sparse)(const asynclm_plan_t*, asynclm_sparse*);
static int (*fn_verify)(const asynclm_draft_rows*, const int32_t*, int32_t, int32_t, const int32_t*, const float*, const float*, int32_t*, int32_t*, void*, void*);
static size_t (*fn_verify_bytes)(int32_t, int32_t);
static PyObject *current_device, *raw_stream;      /* callables: () -> device, (device) -> stream handle */
static PyObject *s_data_ptr, *s_numel, *s_cuda_stream, *s_num_q_heads, *s_num_kv_heads, *s_head_dim, *s_page_size;
/* what a tensor is asked for, and the dtypes of rows, of a quantised cache's tensors and of indices */
static PyObject *s_shape, *s_stride, *s_dtype, *s_is_cuda, *s_is_contiguous, *s_get_device;
static PyObject *t_bf16, *t_e4m3, *t_e8m0, *t_u8, *t_i32, *t_i64, *t_f32;

/* (these return -1 with an exception set on failure) */
static int address(PyObject* tensor, void** out) {
    PyObject* v = PyObject_CallMethodNoArgs(tensor, s_data_ptr);
    if (!v) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

static int address_or_null(PyObject* tensor, void** out) {
    *out = NULL;
    return tensor == Py_None ? 0 : address(tensor, out);
}

static int handle_of(PyObject* v, void** out) {
    *out = v == Py_None ? NULL : PyLong_AsVoidPtr(v);
    return PyErr_Occurred() ? -1 : 0;
}

static int stream_of(PyObject* stream, void** out) {
    PyObject* v;
    if (stream == Py_None) {
        PyObject* device = PyObject_CallNoArgs(current_device);
        if (!device) return -1;
        v = PyObject_CallOneArg(raw_stream, device);
        Py_DECREF(device);
    } else {
        v = PyObject_GetAttr(stream, s_cuda_stream);
    }
    if (!v) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

/* (-1 without an exception where the value does not fit) */
static int int_attr(PyObject* obj, PyObject* name, int32_t* out) {
    PyObject* v = PyObject_GetAttr(obj, name);
    if (!v) return -1;
    const long x = PyLong_AsLong(v);
    Py_DECREF(v);
    *out = (int32_t)x;
    return (x == -1 && PyErr_Occurred()) || x != *out ? -1 : 0;
}

/* A one-dimensional contiguous array of 32-bit integers, held until released; 0 if `obj` is anything else. */
static int int32_array(PyObject* obj, Py_buffer* view) {
    if (PyObject_GetBuffer(obj, view, PyBUF_ND | PyBUF_FORMAT) != 0) {
        PyErr_Clear();
        return 0;
    }
    if (view->ndim == 1 && view->itemsize == 4 && view->format && view->format[0] == 'i' && view->format[1] == 0) return 1;
    PyBuffer_Release(view);
    return 0;
}

static PyObject* py_bind(PyObject* self, PyObject* args) {
    Py_ssize_t plan, append, rope, attn, step;
    PyObject *dev, *raw;
    if (!PyArg_ParseTuple(args, "nnnnnOO", &plan, &append, &rope, &attn, &step, &dev, &raw)) return NULL;
    fn_plan = (void*)plan;
    fn_append = (void*)append;
    fn_append_rope = (void*)rope;
    fn_attn = (void*)attn;
    fn_step = (void*)step;
    Py_XSETREF(current_device, Py_NewRef(dev));
    Py_XSETREF(raw_stream, Py_NewRef(raw));
    Py_RETURN_NONE;
}

/* plan(shape, num_pages, q_indptr, kv_len_before, page_indptr, page_indices, stream, sm_scale, host_ws, dev_ws)
 * -> (status, handle), or None where shape or arrays are not of the kind that needs no conversion. */
static PyObject* py_plan(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 10) return PyErr_Format(PyExc_TypeError, "10 arguments expected");
    asynclm_shape shape = {0};
    if (int_attr(a[0], s_num_q_heads, &shape.num_q_heads) || int_attr(a[0], s_num_kv_heads, &shape.num_kv_heads) ||
        int_attr(a[0], s_head_dim, &shape.head_dim) || int_attr(a[0], s_page_size, &shape.page_size)) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    shape.num_pages = PyLong_AsLongLong(a[1]);
    if (shape.num_pages == -1 && PyErr_Occurred()) return NULL;
    const double scale = PyFloat_AsDouble(a[7]);
    if (scale == -1.0 && PyErr_Occurred()) return NULL;
    shape.sm_scale = (float)scale;
    void *host = NULL, *dev = NULL, *stream = NULL;
    size_t bytes[2];
    if (address(a[8], &host) || address(a[9], &dev) || stream_of(a[6], &stream)) return NULL;
    for (int k = 0; k < 2; ++k) {
        PyObject* v = PyObject_CallMethodNoArgs(a[8 + k], s_numel);
        if (!v) return NULL;
        bytes[k] = PyLong_AsSize_t(v);
        Py_DECREF(v);
        if (PyErr_Occurred()) return NULL;
    }
    Py_buffer view[4];
    int held = 0;
    while (held < 4 && int32_array(a[2 + held], &view[held])) ++held;
    PyObject* result = NULL;
    if (held < 4) {
        result = Py_NewRef(Py_None);
    } else {
        const asynclm_plan_options options = {0};
        const asynclm_batch batch = {(int32_t)view[1].shape[0], view[0].buf, view[1].buf, view[2].buf, view[3].buf};
        asynclm_plan_t* plan = NULL;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = fn_plan(&shape, &options, &batch, host, bytes[0], dev, bytes[1], stream, &plan);
        Py_END_ALLOW_THREADS
        result = Py_BuildValue("(iN)", rc, PyLong_FromVoidPtr(plan));
    }
    while (held > 0) PyBuffer_Release(&view[--held]);
    return result;
}

/* append(handle, k_new, v_new, kv_pool, stream) -> status, and the others alike */
static PyObject* py_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *plan, *k, *v, *pool, *stream;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments expected");
    if (handle_of(a[0], &plan) || address(a[1], &k) || address(a[2], &v) || address(a[3], &pool) || stream_of(a[4], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_append(plan, k, v, pool, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_append_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *plan, *k, *v, *pool, *q, *stream;
    if (n != 7) return PyErr_Format(PyExc_TypeError, "7 arguments expected");
    const double theta = PyFloat_AsDouble(a[5]);
    if (theta == -1.0 && PyErr_Occurred()) return NULL;
    if (handle_of(a[0], &plan) || address(a[1], &k) || address(a[2], &v) || address(a[3], &pool) || address_or_null(a[4], &q) || stream_of(a[6], &stream))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_append_rope(plan, k, v, pool, q, theta, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *plan, *q, *pool, *out, *lse, *stream;
    if (n != 6) return PyErr_Format(PyExc_TypeError, "6 arguments expected");
    if (handle_of(a[0], &plan) || address(a[1], &q) || address(a[2], &pool) || address(a[3], &out) || address_or_null(a[4], &lse) || stream_of(a[5], &stream))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_attn(plan, q, pool, out, lse, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *plan, *q, *k, *v, *pool, *out, *lse, *stream;
    if (n != 8) return PyErr_Format(PyExc_TypeError, "8 arguments expected");
    if (handle_of(a[0], &plan) || address(a[1], &q) || address(a[2], &k) || address(a[3], &v) || address(a[4], &pool) || address(a[5], &out) ||
        address_or_null(a[6], &lse) || stream_of(a[7], &stream))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_step(plan, q, k, v, pool, out, lse, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_bind_kv8(PyObject* self, PyObject* args) {
    Py_ssize_t append, attn, gather, rope, shape;
    PyObject *bf16, *e4m3, *e8m0, *u8, *i32, *i64, *f32;
    if (!PyArg_ParseTuple(args, "nnnnnOOOOOOO", &append, &attn, &gather, &rope, &shape, &bf16, &e4m3, &e8m0, &u8, &i32, &i64, &f32)) return NULL;
    fn_kv8_append = (void*)append;
    fn_kv8_attn = (void*)attn;
    fn_kv8_gather = (void*)gather;
    fn_rope = (void*)rope;
    fn_plan_shape = (void*)shape;
    Py_XSETREF(t_bf16, Py_NewRef(bf16));
    Py_XSETREF(t_e4m3, Py_NewRef(e4m3));
    Py_XSETREF(t_e8m0, Py_NewRef(e8m0));
    Py_XSETREF(t_u8, Py_NewRef(u8));
    Py_XSETREF(t_i32, Py_NewRef(i32));
    Py_XSETREF(t_i64, Py_NewRef(i64));
    Py_XSETREF(t_f32, Py_NewRef(f32));
    Py_RETURN_NONE;
}

/* 1 if the tensor is on a GPU and of one of the two dtypes, 0 if not, -1 with an exception set on failure */
static int is_cuda_of(PyObject* t, PyObject* type, PyObject* or_type) {
    PyObject* v = PyObject_GetAttr(t, s_is_cuda);
    if (!v) return -1;
    const int on = v == Py_True;
    Py_DECREF(v);
    if (!on) return 0;
    v = PyObject_GetAttr(t, s_dtype);
    if (!v) return -1;
    const int right = v == type || v == or_type;
    Py_DECREF(v);
    return right;
}

/* The address of a contiguous tensor of `numel` elements.  1, 0 or -1 as above. */
static int flat(PyObject* t, PyObject* type, PyObject* or_type, Py_ssize_t numel, void** out) {
    const int right = is_cuda_of(t, type, or_type);
    if (right <= 0) return right;
    PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!v) return -1;
    const int whole = v == Py_True;
    Py_DECREF(v);
    if (!whole) return 0;
    v = PyObject_CallMethodNoArgs(t, s_numel);
    if (!v) return -1;
    const Py_ssize_t got = PyLong_AsSsize_t(v);
    Py_DECREF(v);
    if (got == -1 && PyErr_Occurred()) return -1;
    if (got != numel) return 0;
    return address(t, out) ? -1 : 1;
}

/* What a call's tensors have to fit; 0 if there is no such plan. */
typedef struct plan_sizes {
    asynclm_shape shape;
    int32_t batch, tokens;
    Py_ssize_t cache_rows;      /* rows of a quantised cache */
} plan_sizes;
static int sizes_of(const void* plan, plan_sizes* s) {
    if (!plan || fn_plan_shape(plan, &s->shape, &s->batch, &s->tokens) != 0) return 0;
    s->cache_rows = (Py_ssize_t)s->shape.num_pages * 2 * s->shape.num_kv_heads * s->shape.page_size;
    return 1;
}

/* Rows [n][heads][d] of bf16 whose heads lie next to each other and which do not overlap: address, shape and row stride.  (A stride of 0 says "dense" to the C
 * call.)  1, 0 or -1 as above. */
typedef struct rows_view {
    void* ptr;
    Py_ssize_t n, heads, d, stride;
} rows_view;
static int rows_of(PyObject* t, rows_view* r) {
    const int right = is_cuda_of(t, t_bf16, NULL);
    if (right <= 0) return right;
    Py_ssize_t dim[3], step[3];
    for (int which = 0; which < 2; ++which) {
        PyObject* v = which ? PyObject_CallMethodNoArgs(t, s_stride) : PyObject_GetAttr(t, s_shape);
        if (!v) return -1;
        if (!PyTuple_Check(v) || PyTuple_GET_SIZE(v) != 3) {
            Py_DECREF(v);
            return 0;
        }
        for (int k = 0; k < 3; ++k) (which ? step : dim)[k] = PyLong_AsSsize_t(PyTuple_GET_ITEM(v, k));
        Py_DECREF(v);
        if (PyErr_Occurred()) return -1;
    }
    if (dim[0] > 0 && ((dim[2] > 1 && step[2] != 1) || (dim[1] > 1 && step[1] != dim[2]))) return 0;
    if (dim[0] > 1 && step[0] < dim[1] * dim[2]) return 0;
    r->n = dim[0];
    r->heads = dim[1];
    r->d = dim[2];
    r->stride = dim[0] > 1 ? step[0] : 0;
    return address(t, &r->ptr) ? -1 : 1;
}
static int rows_are(const rows_view* r, Py_ssize_t n, Py_ssize_t heads, Py_ssize_t d) { return r->n == n && r->heads == heads && r->d == d; }
static int dense(const rows_view* r) { return r->n <= 1 || r->stride == r->heads * r->d; }

/* The calls of the quantised cache and of rotary rows: status, or None where an argument is not of the kind that needs no conversion
 * or is wrong in a way that the C call cannot see (binding.py says how). `rope`: the address of a table, or 0. */
#define TAKE(x) do { const int got_ = (x); if (got_ < 0) return NULL; if (got_ == 0) Py_RETURN_NONE; } while (0)

/* kv8_append(handle, k_new, v_new, kv8_pool, kv8_scales, rope, q, q_out, stream) */
static PyObject* py_kv8_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "9 arguments expected");
    rows_view k, v, q = {0}, qo = {0};
    void *plan, *pool, *scales, *rope, *stream;
    plan_sizes s;
    if (handle_of(a[0], &plan) || handle_of(a[5], &rope)) return NULL;
    TAKE(sizes_of(plan, &s));
    TAKE(rows_of(a[1], &k));
    TAKE(rows_of(a[2], &v));
    TAKE(rows_are(&k, s.tokens, s.shape.num_kv_heads, s.shape.head_dim) && rows_are(&v, k.n, k.heads, k.d));
    TAKE(flat(a[3], t_e4m3, t_u8, s.cache_rows * s.shape.head_dim, &pool));
    TAKE(flat(a[4], t_e8m0, t_u8, s.cache_rows, &scales));
    if (a[6] != Py_None) {
        if (a[7] == Py_None) Py_RETURN_NONE;
        TAKE(rows_of(a[6], &q));
        TAKE(rows_of(a[7], &qo));
        TAKE(rows_are(&q, s.tokens, s.shape.num_q_heads, s.shape.head_dim) && rows_are(&qo, q.n, q.heads, q.d) && dense(&qo));
    }
    if (stream_of(a[8], &stream)) return NULL;
    const asynclm_kv8_rows rows = {k.ptr, v.ptr, q.ptr, qo.ptr, k.stride, v.stride, q.stride};
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_kv8_append(plan, &rows, pool, scales, rope, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* kv8_attn(handle, q, kv8_pool, kv8_scales, out, lse, stream) */
static PyObject* py_kv8_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "7 arguments expected");
    void *plan, *q, *pool, *scales, *out, *lse = NULL, *stream;
    plan_sizes s;
    if (handle_of(a[0], &plan)) return NULL;
    TAKE(sizes_of(plan, &s));
    const Py_ssize_t rows = (Py_ssize_t)s.tokens * s.shape.num_q_heads;
    TAKE(flat(a[1], t_bf16, NULL, rows * s.shape.head_dim, &q));
    TAKE(flat(a[2], t_e4m3, t_u8, s.cache_rows * s.shape.head_dim, &pool));
    TAKE(flat(a[3], t_e8m0, t_u8, s.cache_rows, &scales));
    TAKE(flat(a[4], t_bf16, NULL, rows * s.shape.head_dim, &out));
    if (a[5] != Py_None) TAKE(flat(a[5], t_f32, NULL, rows, &lse));
    if (stream_of(a[6], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_kv8_attn(plan, q, pool, scales, out, lse, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* kv8_gather(handle, out_indptr, first, kv8_pool, kv8_scales, k_out, v_out, stream) */
static PyObject* py_kv8_gather(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 8) return PyErr_Format(PyExc_TypeError, "8 arguments expected");
    rows_view k, v;
    void *plan, *indptr, *first, *pool, *scales, *stream;
    plan_sizes s;
    if (handle_of(a[0], &plan)) return NULL;
    TAKE(sizes_of(plan, &s));
    TAKE(flat(a[1], t_i64, NULL, (Py_ssize_t)s.batch + 1, &indptr));
    TAKE(flat(a[2], t_i32, NULL, s.batch, &first));
    TAKE(flat(a[3], t_e4m3, t_u8, s.cache_rows * s.shape.head_dim, &pool));
    TAKE(flat(a[4], t_e8m0, t_u8, s.cache_rows, &scales));
    TAKE(rows_of(a[5], &k));
    TAKE(rows_of(a[6], &v));
    TAKE(rows_are(&k, k.n, s.shape.num_kv_heads, s.shape.head_dim) && rows_are(&v, k.n, k.heads, k.d) && dense(&k) && dense(&v));
    if (stream_of(a[7], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_kv8_gather(plan, indptr, first, k.n, pool, scales, k.ptr, v.ptr, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* rope(table, positions, q, q_out, k, k_out, stream) */
static PyObject* py_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "7 arguments expected");
    rows_view in[2], out[2];
    void *table, *positions, *stream;
    if (handle_of(a[0], &table)) return NULL;
    if ((a[4] == Py_None) != (a[5] == Py_None)) Py_RETURN_NONE;
    const int sets = a[4] == Py_None ? 1 : 2;
    asynclm_rope_rows rows[2];
    for (int k = 0; k < sets; ++k) {
        TAKE(rows_of(a[2 + 2 * k], &in[k]));
        TAKE(rows_of(a[3 + 2 * k], &out[k]));
        if (in[k].n != out[k].n || in[k].heads != out[k].heads || in[k].d != out[k].d || in[k].n != in[0].n || in[k].d != in[0].d) Py_RETURN_NONE;
        if (in[k].n > INT32_MAX || in[k].heads > INT32_MAX || in[k].d > INT32_MAX) Py_RETURN_NONE;
        rows[k] = (asynclm_rope_rows){in[k].ptr, out[k].ptr, in[k].stride, out[k].stride, (int32_t)in[k].heads, 0};
    }
    TAKE(flat(a[1], t_i32, NULL, in[0].n, &positions));
    if (stream_of(a[6], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_rope(table, positions, (int32_t)in[0].n, (int32_t)in[0].d, rows, sets, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* kv_bounds(handle, kv_pool, kv8_scales or None, key_bounds, from_start, stream) */
static PyObject* py_bounds(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) return PyErr_Format(PyExc_TypeError, "6 arguments expected");
    void *plan, *pool, *scales = NULL, *bounds, *stream;
    plan_sizes s;
    if (handle_of(a[0], &plan)) return NULL;
    TAKE(sizes_of(plan, &s));
    const int kv8 = a[2] != Py_None;
    TAKE(flat(a[1], kv8 ? t_e4m3 : t_bf16, kv8 ? t_u8 : NULL, s.cache_rows * s.shape.head_dim, &pool));
    if (kv8) TAKE(flat(a[2], t_e8m0, t_u8, s.cache_rows, &scales));
    TAKE(flat(a[3], t_bf16, NULL, (Py_ssize_t)s.shape.num_pages * s.shape.num_kv_heads * 2 * s.shape.head_dim, &bounds));
    const int from_start = PyObject_IsTrue(a[4]);
    if (from_start < 0 || stream_of(a[5], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = kv8 ? fn_kv8_bounds(plan, pool, scales, bounds, from_start, stream) : fn_bounds(plan, pool, bounds, from_start, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* select(handle, q, key_bounds, pages_out or None, stream) */
static PyObject* py_select(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments expected");
    void *plan, *q, *bounds, *out = NULL, *stream;
    plan_sizes s;
    asynclm_sparse sparse;
    if (handle_of(a[0], &plan)) return NULL;
    TAKE(sizes_of(plan, &s));
    TAKE(fn_plan_sparse(plan, &sparse) == 0);
    TAKE(flat(a[1], t_bf16, NULL, (Py_ssize_t)s.tokens * s.shape.num_q_heads * s.shape.head_dim, &q));
    TAKE(flat(a[2], t_bf16, NULL, (Py_ssize_t)s.shape.num_pages * s.shape.num_kv_heads * 2 * s.shape.head_dim, &bounds));
    if (a[3] != Py_None) TAKE(flat(a[3], t_i32, NULL, (Py_ssize_t)s.tokens * s.shape.num_kv_heads * sparse.budget_pages, &out));
    if (stream_of(a[4], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_select(plan, q, bounds, out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* The device of a tensor, or -2 with an exception set on failure. */
static long device_of(PyObject* t) {
    PyObject* v = PyObject_CallMethodNoArgs(t, s_get_device);
    if (!v) return -2;
    const long d = PyLong_AsLong(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -2 : d;
}

/* Rows [n][vocab] of fp32 or bf16 that do not overlap.  1, 0 or -1 as above. */
static int probabilities(PyObject* t, PyObject* type, Py_ssize_t* n, Py_ssize_t* vocab, Py_ssize_t* stride, void** out) {
    const int right = is_cuda_of(t, type, NULL);
    if (right <= 0) return right;
    Py_ssize_t dim[2], step[2];
    for (int which = 0; which < 2; ++which) {
        PyObject* v = which ? PyObject_CallMethodNoArgs(t, s_stride) : PyObject_GetAttr(t, s_shape);
        if (!v) return -1;
        if (!PyTuple_Check(v) || PyTuple_GET_SIZE(v) != 2) {
            Py_DECREF(v);
            return 0;
        }
        for (int k = 0; k < 2; ++k) (which ? step : dim)[k] = PyLong_AsSsize_t(PyTuple_GET_ITEM(v, k));
        Py_DECREF(v);
        if (PyErr_Occurred()) return -1;
    }
    if ((dim[1] > 1 && step[1] != 1) || (dim[0] > 1 && step[0] < dim[1])) return 0;
    *n = dim[0];
    *vocab = dim[1];
    *stride = dim[0] > 1 ? step[0] : dim[1];
    return address(t, out) ? -1 : 1;
}

/* verify(draft_indptr, target, draft or None, draft_tokens, accept_u, sample_u, accepted, tokens_out, workspace, stream); all on the current device */
static PyObject* py_verify(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 10) return PyErr_Format(PyExc_TypeError, "10 arguments expected");
    Py_ssize_t rows, vocab, stride, d_rows = 0, d_vocab = 0, d_stride = 0;
    void *target, *draft = NULL, *p[6], *workspace, *stream;
    PyObject* v = PyObject_GetAttr(a[1], s_dtype);
    if (!v) return NULL;
    PyObject* const type = v == t_f32 ? t_f32 : t_bf16;
    Py_DECREF(v);
    TAKE(probabilities(a[1], type, &rows, &vocab, &stride, &target));
    v = PyObject_CallMethodNoArgs(a[0], s_numel);
    if (!v) return NULL;
    const Py_ssize_t batch = PyLong_AsSsize_t(v) - 1, drafts = rows - batch;
    Py_DECREF(v);
    if (PyErr_Occurred()) return NULL;
    if (batch < 0 || drafts < 0 || batch > INT32_MAX || drafts > INT32_MAX || vocab <= 0 || vocab > INT32_MAX) Py_RETURN_NONE;
    if (a[2] != Py_None) {
        TAKE(probabilities(a[2], type, &d_rows, &d_vocab, &d_stride, &draft));
        if (d_rows != drafts || d_vocab != vocab) Py_RETURN_NONE;
        if (drafts == 0) draft = NULL;
    }
    TAKE(flat(a[0], t_i32, NULL, batch + 1, &p[0]));
    TAKE(flat(a[3], t_i32, NULL, drafts, &p[1]));
    TAKE(flat(a[4], t_f32, NULL, drafts, &p[2]));
    TAKE(flat(a[5], t_f32, NULL, batch, &p[3]));
    TAKE(flat(a[6], t_i32, NULL, batch, &p[4]));
    TAKE(flat(a[7], t_i32, NULL, rows, &p[5]));
    v = PyObject_CallMethodNoArgs(a[8], s_numel);
    if (!v) return NULL;
    const Py_ssize_t bytes = PyLong_AsSsize_t(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) return NULL;
    TAKE(flat(a[8], t_u8, NULL, bytes, &workspace));
    if ((size_t)bytes < fn_verify_bytes((int32_t)batch, (int32_t)vocab)) Py_RETURN_NONE;
    v = PyObject_CallNoArgs(current_device);
    if (!v) return NULL;
    const long device = PyLong_AsLong(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) return NULL;
    for (int k = 0; k < 9; ++k) {
        if (a[k] == Py_None) continue;
        const long d = device_of(a[k]);
        if (d == -2) return NULL;
        if (d != device) Py_RETURN_NONE;
    }
    if (stream_of(a[9], &stream)) return NULL;
    const asynclm_draft_rows r = {target, draft, stride, d_stride, (int32_t)vocab, type == t_f32 ? ASYNCLM_DTYPE_F32 : ASYNCLM_DTYPE_BF16};
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn_verify(&r, p[0], (int32_t)batch, (int32_t)drafts, p[1], p[2], p[3], p[4], p[5], workspace, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_bind_pages(PyObject* self, PyObject* args) {
    Py_ssize_t bounds, kv8_bounds, select, sparse, verify, verify_bytes;
    if (!PyArg_ParseTuple(args, "nnnnnn", &bounds, &kv8_bounds, &select, &sparse, &verify, &verify_bytes)) return NULL;
    fn_bounds = (void*)bounds;
    fn_kv8_bounds = (void*)kv8_bounds;
    fn_select = (void*)select;
    fn_plan_sparse = (void*)sparse;
    fn_verify = (void*)verify;
    fn_verify_bytes = (void*)verify_bytes;
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"bind", py_bind, METH_VARARGS, "bind(plan, append, append_rope, attn, step, current_device, raw_stream)"},
                                {"plan", (PyCFunction)(void*)py_plan, METH_FASTCALL, NULL},
                                {"append", (PyCFunction)(void*)py_append, METH_FASTCALL, NULL},
                                {"append_rope", (PyCFunction)(void*)py_append_rope, METH_FASTCALL, NULL},
                                {"attn", (PyCFunction)(void*)py_attn, METH_FASTCALL, NULL},
                                {"step", (PyCFunction)(void*)py_step, METH_FASTCALL, NULL},
                                {"bind_kv8", py_bind_kv8, METH_VARARGS, "bind_kv8(append, attn, gather, rope, plan_get_shape, bf16, e4m3, e8m0, uint8, int32, int64, float32)"},
                                {"kv8_append", (PyCFunction)(void*)py_kv8_append, METH_FASTCALL, NULL},
                                {"kv8_attn", (PyCFunction)(void*)py_kv8_attn, METH_FASTCALL, NULL},
                                {"kv8_gather", (PyCFunction)(void*)py_kv8_gather, METH_FASTCALL, NULL},
                                {"rope", (PyCFunction)(void*)py_rope, METH_FASTCALL, NULL},
                                {"bind_pages", py_bind_pages, METH_VARARGS, "bind_pages(bounds, kv8_bounds, select_pages, plan_get_sparse, draft_verify, workspace_bytes)"},
                                {"bounds", (PyCFunction)(void*)py_bounds, METH_FASTCALL, NULL},
                                {"select", (PyCFunction)(void*)py_select, METH_FASTCALL, NULL},
                                {"verify", (PyCFunction)(void*)py_verify, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "call_ext", NULL, -1, methods};

PyMODINIT_FUNC PyInit_call_ext(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_num_q_heads = PyUnicode_InternFromString("num_q_heads");
    s_num_kv_heads = PyUnicode_InternFromString("num_kv_heads");
    s_head_dim = PyUnicode_InternFromString("head_dim");
    s_page_size = PyUnicode_InternFromString("page_size");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    if (!s_get_device) return NULL;
    if (!s_shape || !s_stride || !s_dtype || !s_is_cuda || !s_is_contiguous) return NULL;
    if (!s_data_ptr || !s_numel || !s_cuda_stream || !s_num_q_heads || !s_num_kv_heads || !s_head_dim || !s_page_size) return NULL;
    return PyModule_Create(&module);
}
