/* kvs_pycall.c -- argument marshalling of the Python binding, as a CPython extension.
 *
 * Turns the binding's arguments (a geometry, plane addresses, RequestArg / ChunkArg
 * objects) into the C ABI's structs and calls one of its functions by address, with
 * the interpreter lock released.  It takes the ordinary forms only -- exact ints in
 * range, lists and tuples, objects with data_ptr(), contiguous int32 block tables --
 * and returns None, without calling, for anything else: the binding then builds the
 * arguments with numpy, which accepts or refuses them as it always has.
 *
 * What it replaces cost 10 to 16 us for one chunk and 80 us for 128, most of a small
 * call; this takes about 1 us and 25 us.
 *
 * append, attend, weigh (and their forms with axes and sinks) and evict do the same for the model operators' tensors: whatever is not
 * plainly right (a type, a shape, a stride) is left to the binding, which says what is wrong.  Tensors are read
 * by their attributes, or by the reader that use_reader() was given.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include "kvs.h"
#include "kvs_tensor.h"

static PyObject *s_data_ptr, *s_block_table, *s_chunks, *s_first_token, *s_num_tokens, *s_base, *s_residency;

/* 1: *out is the exact int `o`, in [lo, hi]; 0: something else. */
static int small_int(PyObject* o, int64_t lo, int64_t hi, int64_t* out) {
    if (!o || !PyLong_CheckExact(o)) return 0;
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow || v < lo || v > hi) return 0;
    *out = v;
    return 1;
}

/* An address: an exact int, or an object whose data_ptr() returns one.  1 / 0, or -1 with an exception
 * that data_ptr() raised. */
static int address(PyObject* o, uint64_t* out) {
    if (PyLong_CheckExact(o)) {
        const unsigned long long v = PyLong_AsUnsignedLongLong(o);
        if (v == (unsigned long long)-1 && PyErr_Occurred()) {
            PyErr_Clear();
            return 0;
        }
        *out = v;
        return 1;
    }
    PyObject* f = PyObject_GetAttr(o, s_data_ptr);
    if (!f) {
        PyErr_Clear();
        return 0;
    }
    PyObject* r = PyObject_CallNoArgs(f);
    Py_DECREF(f);
    if (!r) return -1;
    int ok = PyLong_CheckExact(r);
    if (ok) {
        *out = PyLong_AsUnsignedLongLong(r);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            ok = 0;
        }
    }
    Py_DECREF(r);
    return ok;
}

static int is_seq(PyObject* o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); }

typedef struct {
    kvs_geometry    geom;
    kvs_paged_cache cache;
    void**          planes;
    kvs_chunk*      chunks;
    kvs_request*    reqs;
    Py_buffer*      tables;
    Py_ssize_t      nreq, nchunk, chunk_cap, nviews;
    void **         ready, **events;
} Args;

static void drop(Args* a) {
    for (Py_ssize_t r = 0; r < a->nviews; ++r) PyBuffer_Release(&a->tables[r]);
    free(a->planes);
    free(a->chunks);
    free(a->reqs);
    free(a->tables);
    free(a->ready);
    free(a->events);
}

static int read_geometry(PyObject* o, kvs_geometry* g) {
    if (PyTuple_CheckExact(o)) {
        int32_t* f[6] = {&g->num_layers, &g->num_kv_heads, &g->head_dim, &g->elem_bytes, &g->block_size, &g->chunk_tokens};
        if (PyTuple_GET_SIZE(o) != 6) return 0;
        for (int k = 0; k < 6; ++k) {
            int64_t v;
            if (!small_int(PyTuple_GET_ITEM(o, k), INT32_MIN, INT32_MAX, &v)) return 0;
            *f[k] = (int32_t)v;
        }
        return 1;
    }
    Py_buffer b;                                             /* a kvs_geometry of the binding */
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return 0;
    }
    const int ok = b.len == (Py_ssize_t)sizeof *g;
    if (ok) memcpy(g, b.buf, sizeof *g);
    PyBuffer_Release(&b);
    return ok;
}

/* Attribute `name` of `o`, held in *held until the next call. */
static PyObject* attr(PyObject* o, PyObject* name, PyObject** held) {
    Py_XDECREF(*held);
    *held = PyObject_GetAttr(o, name);
    if (!*held) PyErr_Clear();
    return *held;
}

/* 1, 0 (not an ordinary request), -1 (exception). */
static int read_request(PyObject* o, Args* a, kvs_request* q) {
    PyObject *held = NULL, *list = NULL, *x;
    int rc = 0;
    int64_t v;
    if (!small_int(attr(o, s_first_token, &held), INT64_MIN, INT64_MAX, &v)) goto out;
    q->first_token = v;
    list = PyObject_GetAttr(o, s_chunks);
    if (!list) PyErr_Clear();
    if (!list || !is_seq(list)) goto out;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    if (a->nchunk + n > a->chunk_cap) {
        const Py_ssize_t cap = (a->nchunk + n) * 2;
        kvs_chunk* grown = realloc(a->chunks, (size_t)cap * sizeof *grown);
        if (!grown) goto out;
        a->chunks = grown;
        a->chunk_cap = cap;
    }
    int64_t sum = 0;
    for (Py_ssize_t k = 0; k < n; ++k) {
        if (k >= PySequence_Fast_GET_SIZE(list)) goto out;   /* data_ptr() may run code that shortens it */
        PyObject* c = PySequence_Fast_GET_ITEM(list, k);
        kvs_chunk* d = &a->chunks[a->nchunk + k];
        uint64_t base;
        Py_INCREF(c);
        x = attr(c, s_base, &held);
        int got = x ? address(x, &base) : 0;
        if (got == 1 && !small_int(attr(c, s_num_tokens, &held), INT32_MIN, INT32_MAX, &v)) got = 0;
        if (got == 1) {
            d->base = (void*)(uintptr_t)base;
            d->num_tokens = (int32_t)v;
            sum += v;
            if (!small_int(attr(c, s_residency, &held), INT32_MIN, INT32_MAX, &v)) got = 0;
            else d->residency = (int32_t)v;
        }
        Py_DECREF(c);
        if (got != 1) {
            rc = got;
            goto out;
        }
    }
    a->nchunk += n;
    q->num_chunks = (int32_t)n;
    x = attr(o, s_num_tokens, &held);
    if (x == Py_None) q->num_tokens = sum;
    else if (small_int(x, INT64_MIN, INT64_MAX, &v)) q->num_tokens = v;
    else goto out;
    x = attr(o, s_block_table, &held);
    Py_buffer* b = &a->tables[a->nviews];
    if (!x) goto out;
    if (PyObject_GetBuffer(x, b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) {
        PyErr_Clear();
        goto out;
    }
    a->nviews++;
    if (b->itemsize != 4 || !b->format || strcmp(b->format, "i") != 0 || b->len / 4 > INT32_MAX) goto out;
    q->block_table = (const int32_t*)b->buf;
    q->block_table_len = (int32_t)(b->len / 4);
    rc = 1;
out:
    Py_XDECREF(held);
    Py_XDECREF(list);
    return rc;
}

/* A list of event handles, or None; 1 / 0. */
static int read_handles(PyObject* o, void*** out) {
    *out = NULL;
    if (o == Py_None) return 1;
    if (!PyList_CheckExact(o)) return 0;
    const Py_ssize_t n = PyList_GET_SIZE(o);
    *out = calloc(n ? (size_t)n : 1, sizeof **out);
    if (!*out) return 0;
    for (Py_ssize_t k = 0; k < n; ++k) {
        uint64_t h;
        if (!PyLong_CheckExact(PyList_GET_ITEM(o, k)) || address(PyList_GET_ITEM(o, k), &h) != 1) return 0;
        (*out)[k] = (void*)(uintptr_t)h;
    }
    return 1;
}

typedef int (*whole_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_request*, int32_t, void*, uint32_t);
typedef int (*layers_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_request*, int32_t, int32_t, void* const*,
                         void*, uint32_t);
typedef int (*store_layers_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_request*, int32_t, int32_t,
                               void* const*, void* const*, void*, uint32_t);

/* call(function, geometry, planes, num_blocks, requests, stream, flags[, kind, layers_per_step, ready, events])
 * -> the status, or None.  kind 1: a layer-wise retrieval, 2: a layer-wise store-back. */
static PyObject* call(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    Args a;
    memset(&a, 0, sizeof a);
    PyObject* result = NULL;
    int64_t fn, nb, stream, flags, kind = 0, lps = 0;
    int got = 0, rc = 0;
    if (nv != 7 && nv != 11) {
        PyErr_SetString(PyExc_TypeError, "call takes 7 or 11 arguments");
        return NULL;
    }
    if (!small_int(v[0], 1, INT64_MAX, &fn) || !read_geometry(v[1], &a.geom) || !is_seq(v[2]) ||
        !small_int(v[3], INT64_MIN, INT64_MAX, &nb) || !is_seq(v[4]) || !small_int(v[5], 0, INT64_MAX, &stream) ||
        !small_int(v[6], 0, UINT32_MAX, &flags))
        goto out;
    if (nv == 11 && (!small_int(v[7], 1, 2, &kind) || !small_int(v[8], INT32_MIN, INT32_MAX, &lps) ||
                     !read_handles(v[9], &a.ready) || !read_handles(v[10], &a.events)))
        goto out;
    const Py_ssize_t np = PySequence_Fast_GET_SIZE(v[2]);
    a.nreq = PySequence_Fast_GET_SIZE(v[4]);
    /* a plane for every layer: the C call reads 2 * num_layers of them */
    if (np == 0 || np < 2 * (Py_ssize_t)a.geom.num_layers || a.nreq > INT32_MAX) goto out;
    a.planes = malloc((size_t)np * sizeof *a.planes);
    a.reqs = calloc((size_t)a.nreq + 1, sizeof *a.reqs);
    a.tables = calloc((size_t)a.nreq + 1, sizeof *a.tables);
    a.chunk_cap = 64;
    a.chunks = malloc((size_t)a.chunk_cap * sizeof *a.chunks);
    if (!a.planes || !a.reqs || !a.tables || !a.chunks) goto out;
    for (Py_ssize_t p = 0; p < np; ++p) {
        uint64_t x;
        if (p >= PySequence_Fast_GET_SIZE(v[2])) goto out;
        PyObject* o = PySequence_Fast_GET_ITEM(v[2], p);
        Py_INCREF(o);
        got = address(o, &x);
        Py_DECREF(o);
        if (got != 1) goto out;
        a.planes[p] = (void*)(uintptr_t)x;
    }
    for (Py_ssize_t r = 0; r < a.nreq; ++r) {
        if (r >= PySequence_Fast_GET_SIZE(v[4])) {
            got = 0;
            goto out;
        }
        PyObject* o = PySequence_Fast_GET_ITEM(v[4], r);
        Py_INCREF(o);
        got = read_request(o, &a, &a.reqs[r]);
        Py_DECREF(o);
        if (got != 1) goto out;
    }
    Py_ssize_t at = 0;                                       /* the chunk array has stopped moving */
    for (Py_ssize_t r = 0; r < a.nreq; ++r) {
        a.reqs[r].chunks = a.chunks + at;
        at += a.reqs[r].num_chunks;
    }
    a.cache.kv_planes = a.planes;
    a.cache.num_blocks = nb;
    got = 1;
    const int32_t n = (int32_t)a.nreq;
    void* s = (void*)(uintptr_t)stream;
    Py_BEGIN_ALLOW_THREADS
    if (kind == 0) rc = ((whole_fn)(uintptr_t)fn)(&a.geom, &a.cache, a.reqs, n, s, (uint32_t)flags);
    else if (kind == 1) rc = ((layers_fn)(uintptr_t)fn)(&a.geom, &a.cache, a.reqs, n, (int32_t)lps, a.events, s, (uint32_t)flags);
    else rc = ((store_layers_fn)(uintptr_t)fn)(&a.geom, &a.cache, a.reqs, n, (int32_t)lps, a.ready, a.events, s, (uint32_t)flags);
    Py_END_ALLOW_THREADS
    result = PyLong_FromLong(rc);
out:
    drop(&a);
    if (result) return result;
    if (got < 0 || PyErr_Occurred()) return NULL;
    Py_RETURN_NONE;
}

/* ---- the model operators ------------------------------------------------- */
static PyObject *s_dtype, *s_shape, *s_stride, *s_cuda_stream, *s_ref;

/* `n` entries of a tuple (or subclass) of ints; 1 / 0. */
static int int_tuple(PyObject* o, int n, int64_t* out) {
    if (!o || !PyTuple_Check(o) || PyTuple_GET_SIZE(o) != n) return 0;
    for (int k = 0; k < n; ++k)
        if (!small_int(PyTuple_GET_ITEM(o, k), 0, INT64_MAX, &out[k])) return 0;
    return 1;
}

typedef kvs_tensor Tensor;

static kvs_read_tensor_fn reader = NULL;                     /* reads a plain tensor without its attributes, where there is one */

/* use_reader(address of a kvs_read_tensor_fn, 0 for none) */
static PyObject* use_reader(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t x;
    if (nv != 1 || !small_int(v[0], 0, INT64_MAX, &x)) {
        PyErr_SetString(PyExc_TypeError, "use_reader takes an address");
        return NULL;
    }
    reader = (kvs_read_tensor_fn)(uintptr_t)x;
    Py_RETURN_NONE;
}

/* A tensor of `dims` dimensions and of that dtype: 1, 0 (something else), -1 (exception). */
static int read_tensor(PyObject* o, PyObject* dtype, int dims, Tensor* t) {
    if (reader) {
        const int got = reader(o, dtype, dims, t);
        if (got != 2) return got;
    }
    PyObject* x = PyObject_GetAttr(o, s_dtype);
    int ok = x == dtype;
    Py_XDECREF(x);
    if (ok) {
        x = PyObject_GetAttr(o, s_shape);
        ok = int_tuple(x, dims, t->shape);
        Py_XDECREF(x);
    }
    if (ok) {
        x = PyObject_CallMethodNoArgs(o, s_stride);
        ok = int_tuple(x, dims, t->stride);
        Py_XDECREF(x);
    }
    if (PyErr_Occurred()) PyErr_Clear();
    return ok ? address(o, &t->at) : 0;
}

typedef struct {
    const kvs_geometry*    geom;
    const kvs_paged_cache* cache;
    const kvs_step*        step;
} StepRef;

/* fn, step (the three structs' addresses), dtype, float32, int32, layer, stream, flags: what every operator begins with. */
enum { V_FN, V_STEP, V_DTYPE, V_F32, V_I32, V_LAYER, V_STREAM, V_FLAGS, V_MORE };

static int read_common(PyObject* const* v, int64_t* fn, StepRef* st, int64_t* layer, int64_t* stream, int64_t* flags) {
    if (!small_int(v[V_FN], 1, INT64_MAX, fn) || !PyBytes_CheckExact(v[V_STEP]) || PyBytes_GET_SIZE(v[V_STEP]) != (Py_ssize_t)sizeof *st ||
        !small_int(v[V_LAYER], INT32_MIN, INT32_MAX, layer) || !small_int(v[V_FLAGS], 0, UINT32_MAX, flags))
        return 0;
    memcpy(st, PyBytes_AS_STRING(v[V_STEP]), sizeof *st);
    *stream = 0;
    if (v[V_STREAM] == Py_None || small_int(v[V_STREAM], 0, INT64_MAX, stream)) return 1;
    PyObject* h = PyObject_GetAttr(v[V_STREAM], s_cuda_stream);
    const int ok = h && small_int(h, 0, INT64_MAX, stream);
    Py_XDECREF(h);
    if (PyErr_Occurred()) PyErr_Clear();
    return ok;
}

/* kvs_rows of a tensor [total_q, heads, head_dim]; *heads 0: any number, which it gets. */
static int read_rows(PyObject* o, PyObject* dtype, const StepRef* st, int64_t* heads, kvs_rows* r) {
    Tensor t;
    const int ok = read_tensor(o, dtype, 3, &t);
    if (ok != 1) return ok;
    if (t.shape[0] != st->step->total_q || t.shape[2] != st->geom->head_dim || t.stride[2] != 1 || t.shape[1] > INT32_MAX ||
        (*heads && t.shape[1] != *heads))
        return 0;
    *heads = t.shape[1];
    r->base = (void*)(uintptr_t)t.at;
    r->row_stride = t.stride[0];
    r->head_stride = t.stride[1];
    return 1;
}

/* A contiguous float32 tensor [total_q, heads]. */
static int read_lse(PyObject* o, PyObject* f32, const StepRef* st, int64_t heads, void** out) {
    Tensor t;
    const int ok = read_tensor(o, f32, 2, &t);
    if (ok != 1) return ok;
    if (t.shape[0] != st->step->total_q || t.shape[1] != heads || (heads > 1 && t.stride[1] != 1) || (t.shape[0] > 1 && t.stride[0] != heads)) return 0;
    *out = (void*)(uintptr_t)t.at;
    return 1;
}

static int read_float(PyObject* o, float* out) {
    if (!PyFloat_CheckExact(o)) return 0;
    *out = (float)PyFloat_AS_DOUBLE(o);
    return 1;
}

static int read_bool(PyObject* o, int32_t* out) {
    *out = o == Py_True;
    return o == Py_True || o == Py_False;
}

typedef int (*op_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_step*, int32_t, const void*, void*, uint32_t);

static PyObject* run_op(int got, int64_t fn, const StepRef* st, int64_t layer, const void* args, int64_t stream, int64_t flags) {
    if (got < 0) return NULL;
    if (got == 0) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((op_fn)(uintptr_t)fn)(st->geom, st->cache, st->step, (int32_t)layer, args, (void*)(uintptr_t)stream, (uint32_t)flags);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*sinks_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_step*, int32_t, const void*, int32_t, void*, uint32_t);

static PyObject* run_sinks_op(int got, int64_t fn, const StepRef* st, int64_t layer, const void* args, int64_t sinks, int64_t stream, int64_t flags) {
    if (got < 0) return NULL;
    if (got == 0) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((sinks_fn)(uintptr_t)fn)(st->geom, st->cache, st->step, (int32_t)layer, args, (int32_t)sinks, (void*)(uintptr_t)stream, (uint32_t)flags);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

#define TRY(call)                   \
    do {                            \
        if (got == 1) got = (call); \
    } while (0)

/* The struct behind an object's ref (its address); 1 / 0. */
static int read_ref(PyObject* o, const void** out) {
    int64_t x = 0;
    PyObject* ref = PyObject_GetAttr(o, s_ref);
    const int ok = ref && small_int(ref, 1, INT64_MAX, &x);
    Py_XDECREF(ref);
    if (PyErr_Occurred()) PyErr_Clear();
    *out = (const void*)(uintptr_t)x;
    return ok;
}

/* q, k, v, q_out, rope */
static int read_append(PyObject* const* v, const StepRef* st, int got, kvs_append_args* a) {
    PyObject* const* w = v + V_MORE;
    int64_t heads = 0;
    if (w[0] != Py_None) {
        TRY(read_rows(w[0], v[V_DTYPE], st, &heads, &a->q));
        a->num_q_heads = (int32_t)heads;
        if (w[3] == Py_None) a->q_out = a->q;
        else TRY(read_rows(w[3], v[V_DTYPE], st, &heads, &a->q_out));
    }
    int64_t H = got == 1 ? st->geom->num_kv_heads : 1;
    TRY(read_rows(w[1], v[V_DTYPE], st, &H, &a->k));
    TRY(read_rows(w[2], v[V_DTYPE], st, &H, &a->v));
    if (w[4] != Py_None) {
        const void* p = NULL;
        TRY(read_ref(w[4], &p));
        a->rope = (const kvs_rope*)p;
    }
    return got;
}

/* ..., q, k, v, q_out, rope, positions */
static PyObject* append(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags;
    StepRef st;
    kvs_append_args a;
    memset(&a, 0, sizeof a);
    if (nv != V_MORE + 6) {
        PyErr_SetString(PyExc_TypeError, "append takes 14 arguments");
        return NULL;
    }
    int got = read_append(v, &st, read_common(v, &fn, &st, &layer, &stream, &flags), &a);
    PyObject* positions = v[V_MORE + 5];
    if (positions != Py_None) {
        Tensor t;
        TRY(read_tensor(positions, v[V_I32], 1, &t));
        if (got == 1) {
            got = t.shape[0] == st.step->total_q && (t.shape[0] <= 1 || t.stride[0] == 1);
            a.positions = (const int32_t*)(uintptr_t)t.at;
        }
    }
    return run_op(got, fn, &st, layer, &a, stream, flags);
}

typedef int (*axes_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_step*, int32_t, const void*, const kvs_axes*, void*, uint32_t);

/* ..., q, k, v, q_out, rope, axes, positions */
static PyObject* append_axes(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags;
    StepRef st;
    kvs_append_args a;
    kvs_axes x;
    memset(&a, 0, sizeof a);
    memset(&x, 0, sizeof x);
    if (nv != V_MORE + 7) {
        PyErr_SetString(PyExc_TypeError, "append_axes takes 15 arguments");
        return NULL;
    }
    int got = read_append(v, &st, read_common(v, &fn, &st, &layer, &stream, &flags), &a);
    PyObject* const* w = v + V_MORE;
    const void* p = NULL;
    Tensor t;
    if (w[4] == Py_None) got = got < 0 ? got : 0;
    TRY(read_ref(w[5], &p));
    if (got == 1) memcpy(&x, p, sizeof x);
    TRY(read_tensor(w[6], v[V_I32], 2, &t));
    if (got == 1) {
        got = t.shape[0] == x.num_axes && t.shape[1] == st.step->total_q && (t.shape[1] <= 1 || t.stride[1] == 1);
        a.positions = (const int32_t*)(uintptr_t)t.at;
        x.stride = t.stride[0];
    }
    if (got < 0) return NULL;
    if (got == 0) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((axes_fn)(uintptr_t)fn)(st.geom, st.cache, st.step, (int32_t)layer, &a, &x, (void*)(uintptr_t)stream, (uint32_t)flags);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* q, out, lse, scale, causal, window */
static int read_attend(PyObject* const* v, const StepRef* st, int got, kvs_attend_args* a) {
    PyObject* const* w = v + V_MORE;
    int64_t heads = 0, window = 0;
    TRY(read_rows(w[0], v[V_DTYPE], st, &heads, &a->q));
    TRY(read_rows(w[1], v[V_DTYPE], st, &heads, &a->out));
    if (w[2] != Py_None) {
        void* p = NULL;
        TRY(read_lse(w[2], v[V_F32], st, heads, &p));
        a->lse = (float*)p;
    }
    TRY(read_float(w[3], &a->scale));
    TRY(read_bool(w[4], &a->causal));
    TRY(small_int(w[5], INT32_MIN, INT32_MAX, &window));
    a->window = (int32_t)window;
    a->num_q_heads = (int32_t)heads;
    return got;
}

static int read_workspace(PyObject* o, PyObject* byte, kvs_attend_args* a) {
    Tensor t;
    if (o == Py_None) return 1;
    const int ok = read_tensor(o, byte, 1, &t);
    if (ok != 1) return ok;
    a->workspace = (void*)(uintptr_t)t.at;
    a->workspace_bytes = t.shape[0];
    return t.stride[0] == 1 || t.shape[0] <= 1;
}

/* ..., q, out, lse, scale, causal, window, workspace, uint8 */
static PyObject* attend(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags;
    StepRef st;
    kvs_attend_args a;
    memset(&a, 0, sizeof a);
    if (nv != V_MORE + 8) {
        PyErr_SetString(PyExc_TypeError, "attend takes 16 arguments");
        return NULL;
    }
    int got = read_attend(v, &st, read_common(v, &fn, &st, &layer, &stream, &flags), &a);
    TRY(read_workspace(v[V_MORE + 6], v[V_MORE + 7], &a));
    return run_op(got, fn, &st, layer, &a, stream, flags);
}

/* ..., q, out, lse, scale, causal, window, sinks, workspace, uint8 */
static PyObject* attend_sinks(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags, sinks = 0;
    StepRef st;
    kvs_attend_args a;
    memset(&a, 0, sizeof a);
    if (nv != V_MORE + 9) {
        PyErr_SetString(PyExc_TypeError, "attend_sinks takes 17 arguments");
        return NULL;
    }
    int got = read_attend(v, &st, read_common(v, &fn, &st, &layer, &stream, &flags), &a);
    TRY(small_int(v[V_MORE + 6], INT32_MIN, INT32_MAX, &sinks));
    TRY(read_workspace(v[V_MORE + 7], v[V_MORE + 8], &a));
    return run_sinks_op(got, fn, &st, layer, &a, sinks, stream, flags);
}

/* q, lse, weights, scale, decay, causal, window */
static int read_weigh(PyObject* const* v, const StepRef* st, int got, kvs_weigh_args* a) {
    PyObject* const* w = v + V_MORE;
    int64_t heads = 0, window = 0;
    void* p = NULL;
    Tensor t;
    TRY(read_rows(w[0], v[V_DTYPE], st, &heads, &a->q));
    TRY(read_lse(w[1], v[V_F32], st, heads, &p));
    TRY(read_tensor(w[2], v[V_F32], 3, &t));
    if (got == 1) {
        got = t.shape[0] == st->step->num_requests && t.shape[1] == st->geom->num_kv_heads && t.shape[2] >= st->step->max_kv && t.stride[2] == 1;
        a->weights = (float*)(uintptr_t)t.at;
        a->request_stride = t.stride[0];
        a->head_stride = t.stride[1];
    }
    TRY(read_float(w[3], &a->scale));
    TRY(read_float(w[4], &a->decay));
    TRY(read_bool(w[5], &a->causal));
    TRY(small_int(w[6], INT32_MIN, INT32_MAX, &window));
    a->lse = (const float*)p;
    a->window = (int32_t)window;
    a->num_q_heads = (int32_t)heads;
    return got;
}

/* ..., q, lse, weights, scale, decay, causal, window */
static PyObject* weigh(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags;
    StepRef st;
    kvs_weigh_args a;
    memset(&a, 0, sizeof a);
    if (nv != V_MORE + 7) {
        PyErr_SetString(PyExc_TypeError, "weigh takes 15 arguments");
        return NULL;
    }
    const int got = read_weigh(v, &st, read_common(v, &fn, &st, &layer, &stream, &flags), &a);
    return run_op(got, fn, &st, layer, &a, stream, flags);
}

/* ..., q, lse, weights, scale, decay, causal, window, sinks */
static PyObject* weigh_sinks(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags, sinks = 0;
    StepRef st;
    kvs_weigh_args a;
    memset(&a, 0, sizeof a);
    if (nv != V_MORE + 8) {
        PyErr_SetString(PyExc_TypeError, "weigh_sinks takes 16 arguments");
        return NULL;
    }
    int got = read_weigh(v, &st, read_common(v, &fn, &st, &layer, &stream, &flags), &a);
    TRY(small_int(v[V_MORE + 7], INT32_MIN, INT32_MAX, &sinks));
    return run_sinks_op(got, fn, &st, layer, &a, sinks, stream, flags);
}

typedef int (*evict_fn)(const kvs_geometry*, const kvs_paged_cache*, const kvs_step*, const kvs_evict_args*, void*, uint32_t);

static int contiguous(const Tensor* t, int dims) {
    int64_t n = 1;
    for (int k = dims - 1; k >= 0; --k) {
        if (t->shape[k] > 1 && t->stride[k] != n) return 0;
        n *= t->shape[k];
    }
    return 1;
}

/* ..., weights, dst_tables, budget, sinks, recent, kept, new_weights, new_lens (the layer is not used) */
static PyObject* evict(PyObject* self, PyObject* const* v, Py_ssize_t nv) {
    (void)self;
    int64_t fn, layer, stream, flags, budget = 0, sinks = 0, recent = 0;
    StepRef st;
    kvs_evict_args a;
    memset(&a, 0, sizeof a);
    if (nv != V_MORE + 8) {
        PyErr_SetString(PyExc_TypeError, "evict takes 16 arguments");
        return NULL;
    }
    int got = read_common(v, &fn, &st, &layer, &stream, &flags);
    PyObject* const* w = v + V_MORE;
    Tensor t;
    memset(&t, 0, sizeof t);
    const int64_t L = got == 1 ? st.geom->num_layers : 0, H = got == 1 ? st.geom->num_kv_heads : 0, R = got == 1 ? st.step->num_requests : 0;
    TRY(small_int(w[2], 1, INT32_MAX, &budget));
    TRY(small_int(w[3], INT32_MIN, INT32_MAX, &sinks));
    TRY(small_int(w[4], INT32_MIN, INT32_MAX, &recent));
    TRY(read_tensor(w[0], v[V_F32], 4, &t));
    if (got == 1) {
        got = t.shape[0] == L && t.shape[1] == R && t.shape[2] == H && t.shape[3] >= st.step->max_kv && t.stride[3] == 1;
        a.weights = (const float*)(uintptr_t)t.at;
        a.layer_stride = t.stride[0];
        a.request_stride = t.stride[1];
        a.head_stride = t.stride[2];
    }
    TRY(read_tensor(w[1], v[V_I32], 2, &t));
    if (got == 1) {
        const int64_t most = st.step->max_kv < budget ? st.step->max_kv : budget;
        got = t.shape[0] == R && t.stride[1] == 1 && (R <= 1 || t.stride[0] >= t.shape[1]) && t.shape[1] <= INT32_MAX && t.stride[0] <= INT32_MAX &&
              t.shape[1] * st.geom->block_size >= most;
        a.dst_tables = (const int32_t*)(uintptr_t)t.at;
        a.dst_stride = (int32_t)(R > 1 ? t.stride[0] : t.shape[1]);
    }
    TRY(read_tensor(w[5], v[V_I32], 4, &t));
    if (got == 1) {
        got = t.shape[0] == L && t.shape[1] == R && t.shape[2] == H && t.shape[3] == budget && contiguous(&t, 4);
        a.kept = (int32_t*)(uintptr_t)t.at;
    }
    if (w[6] != Py_None) {
        TRY(read_tensor(w[6], v[V_F32], 4, &t));
        if (got == 1) {
            got = t.shape[0] == L && t.shape[1] == R && t.shape[2] == H && t.shape[3] == budget && contiguous(&t, 4);
            a.new_weights = (float*)(uintptr_t)t.at;
        }
    }
    if (w[7] != Py_None) {
        TRY(read_tensor(w[7], v[V_I32], 1, &t));
        if (got == 1) {
            got = t.shape[0] == R && contiguous(&t, 1);
            a.new_lens = (int32_t*)(uintptr_t)t.at;
        }
    }
    a.budget = (int32_t)budget;
    a.sinks = (int32_t)sinks;
    a.recent = (int32_t)recent;
    if (got < 0) return NULL;
    if (got == 0) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((evict_fn)(uintptr_t)fn)(st.geom, st.cache, st.step, &a, (void*)(uintptr_t)stream, (uint32_t)flags);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(call), METHOD(append), METHOD(append_axes), METHOD(attend), METHOD(attend_sinks),
                                METHOD(weigh), METHOD(weigh_sinks), METHOD(evict), METHOD(use_reader), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "kvs_pycall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit_kvs_pycall(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_block_table = PyUnicode_InternFromString("block_table");
    s_chunks = PyUnicode_InternFromString("chunks");
    s_first_token = PyUnicode_InternFromString("first_token");
    s_num_tokens = PyUnicode_InternFromString("num_tokens");
    s_base = PyUnicode_InternFromString("base");
    s_residency = PyUnicode_InternFromString("residency");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_ref = PyUnicode_InternFromString("ref");
    return PyModule_Create(&module);
}
