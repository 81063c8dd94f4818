/* The Python side's calls that are made once per layer and token, as vectorcall functions: ctypes converts eight arguments
 * in 1.1 us, a quarter of what such a call costs on the host; this takes 0.2.  Every function gets the address of the
 * library's entry point first (so it follows whichever build of the library is loaded) and then that entry point's arguments
 * as numbers, None for a null pointer, or as tensors.  The status comes back as an int; the GIL is released around the call. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

/* What ctypes takes for a number or an address besides an int: one of its own simple values (a handle or stream kept as a
 * c_void_p, say) and anything with _as_parameter_.  A new reference, or NULL with the error set. */
static PyObject* plain(PyObject* o) {
    static PyObject* simple = NULL;
    PyObject* v = PyObject_GetAttrString(o, "_as_parameter_");
    if (v != NULL) return v;
    PyErr_Clear();
    if (simple == NULL) {
        PyObject* m = PyImport_ImportModule("ctypes");
        simple = m != NULL ? PyObject_GetAttrString(m, "_SimpleCData") : NULL;
        Py_XDECREF(m);
        if (simple == NULL) return NULL;
    }
    switch (PyObject_IsInstance(o, simple)) {
        case 1: return PyObject_GetAttrString(o, "value");
        case 0: PyErr_Format(PyExc_TypeError, "an int or None, not %.80s", Py_TYPE(o)->tp_name);
    }
    return NULL;
}

/* kind 'p': an address, or None for a null pointer; 'i': an integer.  Kept out of the converters, which are inlined. */
static __attribute__((noinline)) int from_other(PyObject* o, char kind, void** ptr, int64_t* i64) {
    PyObject* v = plain(o);
    int ok = v != NULL;
    if (ok && kind == 'p' && v == Py_None) *ptr = NULL;
    else if (ok && PyLong_Check(v)) {
        if (kind == 'p') *ptr = PyLong_AsVoidPtr(v);
        else *i64 = PyLong_AsLongLong(v);
        ok = !PyErr_Occurred();
    } else if (ok) {
        PyErr_Format(PyExc_TypeError, "an int or None, not %.80s", Py_TYPE(o)->tp_name);
        ok = 0;
    }
    Py_XDECREF(v);
    return ok;
}
static int as_ptr(PyObject* o, void** out) {
    if (o == Py_None) { *out = NULL; return 1; }
    if (!PyLong_Check(o)) return from_other(o, 'p', out, NULL);
    *out = PyLong_AsVoidPtr(o);
    return !(*out == NULL && PyErr_Occurred());
}
static int as_i64(PyObject* o, int64_t* out) {
    if (!PyLong_Check(o)) return from_other(o, 'i', NULL, out);
    *out = PyLong_AsLongLong(o);
    return !(*out == -1 && PyErr_Occurred());
}
static int as_int(PyObject* o, int* out) {
    int64_t v;
    if (!as_i64(o, &v)) return 0;
    if (v != (int64_t)(int)v) { PyErr_SetString(PyExc_OverflowError, "argument does not fit a C int"); return 0; }
    *out = (int)v;
    return 1;
}
static int as_float(PyObject* o, float* out) {
    const double v = PyFloat_AsDouble(o);
    *out = (float)v;
    return !(v == -1.0 && PyErr_Occurred());
}
static int count(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return 1;
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
    return 0;
}

typedef int (*spmspv_fn)(void*, const void*, int, float, const void*, void*, int, void*);
static PyObject* call_spmspv(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *h, *x, *mask, *y, *stream;
    int rule, ydt, st;
    float thr;
    if (!count(n, 9) || !as_ptr(a[0], &f) || !as_ptr(a[1], &h) || !as_ptr(a[2], &x) || !as_int(a[3], &rule) || !as_float(a[4], &thr) ||
        !as_ptr(a[5], &mask) || !as_ptr(a[6], &y) || !as_int(a[7], &ydt) || !as_ptr(a[8], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((spmspv_fn)f)(h, x, rule, thr, mask, y, ydt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*batch_fn)(void*, const void*, int64_t, int, int, float, const void*, int64_t, void*, int64_t, int, void*);
static PyObject* call_spmspv_batch(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *h, *x, *mask, *y, *stream;
    int64_t ldx, mstride, ldy;
    int batch, rule, ydt, st;
    float thr;
    if (!count(n, 13) || !as_ptr(a[0], &f) || !as_ptr(a[1], &h) || !as_ptr(a[2], &x) || !as_i64(a[3], &ldx) || !as_int(a[4], &batch) ||
        !as_int(a[5], &rule) || !as_float(a[6], &thr) || !as_ptr(a[7], &mask) || !as_i64(a[8], &mstride) || !as_ptr(a[9], &y) ||
        !as_i64(a[10], &ldy) || !as_int(a[11], &ydt) || !as_ptr(a[12], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((batch_fn)f)(h, x, ldx, batch, rule, thr, mask, mstride, y, ldy, ydt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*spmm_fn)(void*, const void*, int64_t, int64_t, void*, int64_t, int, void*);
static PyObject* call_spmm(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *h, *x, *y, *stream;
    int64_t rows, ldx, ldy;
    int ydt, st;
    if (!count(n, 9) || !as_ptr(a[0], &f) || !as_ptr(a[1], &h) || !as_ptr(a[2], &x) || !as_i64(a[3], &rows) || !as_i64(a[4], &ldx) ||
        !as_ptr(a[5], &y) || !as_i64(a[6], &ldy) || !as_int(a[7], &ydt) || !as_ptr(a[8], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((spmm_fn)f)(h, x, rows, ldx, y, ldy, ydt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*swiglu_fn)(const void*, const void*, int64_t, float, void*, void*, void*, void*);
static PyObject* call_swiglu_dp(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *gate, *up, *x, *mask, *cnt, *stream;
    int64_t k;
    float thr;
    int st;
    if (!count(n, 9) || !as_ptr(a[0], &f) || !as_ptr(a[1], &gate) || !as_ptr(a[2], &up) || !as_i64(a[3], &k) || !as_float(a[4], &thr) ||
        !as_ptr(a[5], &x) || !as_ptr(a[6], &mask) || !as_ptr(a[7], &cnt) || !as_ptr(a[8], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((swiglu_fn)f)(gate, up, k, thr, x, mask, cnt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* The calls around the projections take torch tensors: eight of them, looked at from Python, cost 4 us of such a call's 8, from here
 * a tenth of that.  What follows is the part of DLPack's exchange table (version 1.3, the attribute __dlpack_c_exchange_api__ of
 * a tensor's type) that this takes. */
typedef struct {
    void* data;
    int32_t device_type, device_id;
    int32_t ndim;
    uint8_t code, bits;
    uint16_t lanes;
    int64_t* shape;
    int64_t* strides;
    uint64_t byte_offset;
} dl_tensor;
typedef struct {
    uint32_t major, minor;
    void* older;
    void* managed[3];
    int (*look)(void*, dl_tensor*);
    int (*stream)(int32_t, int32_t, void**);
} dl_table;
enum { DL_CPU = 1, DL_CUDA = 2, MOST_DIMS = 3 };
typedef enum { OTHER, F16, F32, I32, U32, I64, U8 } kind_t;

typedef struct {
    char* p;
    int64_t size[MOST_DIMS], step[MOST_DIMS];
    int ndim, device;                           /* device: as get_device() has it, -1 for the host's memory */
    kind_t kind;
} tensor;

static const dl_table* table_of(PyObject* o, const char* name) {
    static PyTypeObject* known = NULL;
    static const dl_table* its = NULL;
    PyTypeObject* type = Py_TYPE(o);
    if (type == known) return its;
    PyObject* capsule = PyObject_GetAttrString((PyObject*)type, "__dlpack_c_exchange_api__");
    if (capsule == NULL) {
        PyErr_Clear();
        PyErr_Format(PyExc_TypeError, "%s must be a torch tensor (of a PyTorch with __dlpack_c_exchange_api__), not %.80s", name, type->tp_name);
        return NULL;
    }
    const dl_table* t = (const dl_table*)PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
    Py_DECREF(capsule);
    if (t == NULL) return NULL;
    if (t->major != 1 || t->look == NULL || t->stream == NULL) {
        PyErr_SetString(PyExc_RuntimeError, "this PyTorch's __dlpack_c_exchange_api__ is not of version 1");
        return NULL;
    }
    Py_INCREF(type);                            /* so that no other type gets its address */
    Py_XDECREF(known);
    known = type, its = t;
    return t;
}

static int look(PyObject* o, const char* name, tensor* t) {
    dl_tensor d;
    const dl_table* table = table_of(o, name);
    if (table == NULL) return 0;
    if (table->look(o, &d) != 0) {
        if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s cannot be looked at", name);
        return 0;
    }
    if (d.ndim > MOST_DIMS) {
        PyErr_Format(PyExc_ValueError, "%s has %d dimensions", name, (int)d.ndim);
        return 0;
    }
    t->p = (char*)d.data + d.byte_offset;
    t->ndim = d.ndim;
    t->device = d.device_type == DL_CUDA ? d.device_id : d.device_type == DL_CPU ? -1 : -3;
    t->kind = d.lanes != 1 ? OTHER : d.code == 2 ? (d.bits == 16 ? F16 : d.bits == 32 ? F32 : OTHER) : d.code == 0 ? (d.bits == 32 ? I32 : d.bits == 64 ? I64 : OTHER) :
              d.code == 1 ? (d.bits == 8 ? U8 : d.bits == 32 ? U32 : OTHER) : OTHER;
    int64_t dense = 1;
    for (int i = d.ndim - 1; i >= 0; --i) {
        t->size[i] = d.shape[i];
        t->step[i] = d.strides != NULL ? d.strides[i] : dense;
        dense *= d.shape[i];
    }
    return 1;
}

static int refuse(const char* what) { PyErr_SetString(PyExc_ValueError, what); return 0; }

static int contiguous(const tensor* t) {
    int64_t dense = 1;
    for (int i = t->ndim - 1; i >= 0; --i) {
        if (t->size[i] == 0) return 1;
        if (t->size[i] != 1 && t->step[i] != dense) return 0;
        dense *= t->size[i];
    }
    return 1;
}

static int64_t numel(const tensor* t) {
    int64_t n = 1;
    for (int i = 0; i < t->ndim; ++i) n *= t->size[i];
    return n;
}

/* A contiguous vector of n values (n < 0: as many as it has, left in *count); None stays a null pointer. */
static int vector(PyObject* o, kind_t kind, const char* dtype, int64_t n, int64_t* count, const char* name, int here, void** p) {
    tensor t;
    *p = NULL;
    if (o == Py_None) return 1;
    if (!look(o, name, &t)) return 0;
    if (n < 0) n = *count = numel(&t);
    if (t.kind != kind || t.device != here || !contiguous(&t) || numel(&t) != n) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous CUDA %s of %lld values on the current device", name, dtype, (long long)n);
        return 0;
    }
    *p = t.p;
    return 1;
}

/* [n][m] whose rows are contiguous: *ld elements between them. */
static int rows(const tensor* t, int64_t n, int64_t m, const char* name, int here, int64_t* ld) {
    if (t->ndim != 2 || t->size[0] != n || t->size[1] != m || t->device != here) {
        PyErr_Format(PyExc_ValueError, "%s must be CUDA [%lld][%lld] on the current device", name, (long long)n, (long long)m);
        return 0;
    }
    if (t->step[1] != 1 && m > 1) {
        PyErr_Format(PyExc_ValueError, "the last dimension of %s must be contiguous", name);
        return 0;
    }
    *ld = n > 1 || t->step[0] > m ? t->step[0] : m;
    return 1;
}

/* [n][heads][dim] whose heads lie one after another: *ld elements between tokens. */
static int heads(const tensor* t, int64_t n, int64_t count, int64_t dim, const char* name, int here, int64_t* ld) {
    if (t->ndim != 3 || t->size[0] != n || t->size[1] != count || t->size[2] != dim || t->device != here) {
        PyErr_Format(PyExc_ValueError, "%s must be CUDA [%lld][%lld][%lld] on the current device", name, (long long)n, (long long)count, (long long)dim);
        return 0;
    }
    if ((t->step[2] != 1 && dim > 1) || (t->step[1] != dim && count > 1)) {
        PyErr_Format(PyExc_ValueError, "the heads of a token of %s must be contiguous", name);
        return 0;
    }
    *ld = n > 1 || t->step[0] > count * dim ? t->step[0] : count * dim;
    return 1;
}

/* `like`: any of the call's tensors. */
static int stream_of(PyObject* o, PyObject* like, int here, void** stream) {
    if (o == Py_None) {
        const dl_table* table = table_of(like, "tensor");
        if (table == NULL) return 0;
        if (table->stream(DL_CUDA, here, stream) == 0) return 1;
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "no current stream");
        return 0;
    }
    if (PyLong_Check(o)) return as_ptr(o, stream);
    PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
    if (v == NULL) {
        PyErr_Clear();
        return as_ptr(o, stream);
    }
    const int ok = as_ptr(v, stream);
    Py_DECREF(v);
    return ok;
}

/* A row as a matrix of one. */
static void as_rows(tensor* t) {
    if (t->ndim != 1) return;
    t->size[1] = t->size[0], t->step[1] = t->step[0];
    t->size[0] = 1, t->step[0] = t->size[1], t->ndim = 2;
}

typedef int (*lora_fn)(const void*, int64_t, int64_t, int64_t, const void*, const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, int,
                       const void*, const void*, const void*, int64_t, void*, int64_t, int64_t, int, void*);
/* the device, X, adapter, A, B, Y, base (None: Y), scales, ranks, stream */
static PyObject* call_lora(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *adapter, *ranks, *scales, *stream;
    int64_t ldx, ldy, ldbase, lda, ldb;
    int here, st;
    tensor x, wa, wb, y, base;
    if (!count(n, 11) || !as_ptr(a[0], &f) || !as_int(a[1], &here)) return NULL;
    PyObject* from = a[7] == Py_None ? a[6] : a[7];
    if (!look(a[2], "X", &x) || !look(a[4], "A", &wa) || !look(a[5], "B", &wb) || !look(a[6], "Y", &y) || !look(from, "base", &base)) return NULL;
    if (x.ndim == 1) as_rows(&x), as_rows(&y), as_rows(&base);
    if (x.ndim != 2 || wa.ndim != 3 || wb.ndim != 3 || wa.size[2] != x.size[1] || wb.size[0] != wa.size[0] || wb.size[2] != wa.size[1]) {
        refuse("X must be [N][K], A [count][rank][K] and B [count][M][rank]");
        return NULL;
    }
    const int64_t N = x.size[0], K = x.size[1], rank = wa.size[1], M = wb.size[1], adapters = wa.size[0];
    if (x.kind != F16 || wa.kind != F16 || wb.kind != F16 || (y.kind != F16 && y.kind != F32) || base.kind != y.kind) {
        refuse("X, A and B must be fp16, Y and base both fp16 or both fp32");
        return NULL;
    }
    if (wa.device != here || wb.device != here || (wa.step[2] != 1 && K > 1) || (wb.step[2] != 1 && rank > 1)) {
        refuse("A and B must be CUDA tensors on the current device with a contiguous last dimension");
        return NULL;
    }
    if (a[3] == Py_None) {
        refuse("adapter is required");
        return NULL;
    }
    lda = rank > 1 || wa.step[1] > K ? wa.step[1] : K, ldb = M > 1 || wb.step[1] > rank ? wb.step[1] : rank;
    if (!rows(&x, N, K, "X", here, &ldx) || !rows(&y, N, M, "Y", here, &ldy) || !rows(&base, N, M, "base", here, &ldbase) ||
        !vector(a[3], I32, "int32", N, NULL, "adapter", here, &adapter) || !vector(a[8], F32, "float32", adapters, NULL, "scales", here, &scales) ||
        !vector(a[9], I32, "int32", adapters, NULL, "ranks", here, &ranks) || !stream_of(a[10], a[2], here, &stream))
        return NULL;
    if (rank > INT32_MAX) { refuse("rank is beyond 32 bits"); return NULL; }
    Py_BEGIN_ALLOW_THREADS
    st = ((lora_fn)f)(x.p, N, K, ldx, adapter, wa.p, lda, wa.step[0], wb.p, ldb, wb.step[0], adapters, (int)rank, ranks, scales, base.p, ldbase, y.p, M, ldy,
                      y.kind == F32, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

#define MOST_AXES 4
/* The sections come as a sequence of ints, one for each axis, or None (one axis has all pairs). */
static int sections_of(PyObject* o, int64_t axes, int64_t pairs, int* out) {
    if (o == Py_None && axes == 1) {
        out[0] = (int)pairs;
        return 1;
    }
    PyObject* s = o == Py_None ? NULL : PySequence_Fast(o, "sections: a sequence of one int for each axis");
    int ok = s != NULL && PySequence_Fast_GET_SIZE(s) == axes;
    if (!ok && !PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "sections: a sequence of one int for each axis");
    for (int i = 0; ok && i < axes && i < MOST_AXES; ++i) ok = as_int(PySequence_Fast_GET_ITEM(s, i), &out[i]);
    Py_XDECREF(s);
    return ok;
}

typedef int (*heads_fn)(const void*, int64_t, const void*, int64_t, int, int64_t, int, int, int, const void*, const void*, float, const void*, int64_t, int,
                        const int*, const void*, int, int, void*, int64_t, void*, int64_t, void*);
/* the device, q, k (may be None, with k_out), q_out, k_out, pos, inv_freq (None: no rotation), sections, q_weight, k_weight, eps, adjacent, stream */
static PyObject* call_qk_norm_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *qw, *kw = NULL, *freq = NULL, *stream;
    int64_t ldq, ldk = 0, ldq_out, ldk_out = 0, pairs = 0, axes = 0, pos_stride = 0;
    int here, adjacent, st, sections[MOST_AXES] = {0};
    float eps;
    tensor q, k = {0}, q_out, k_out = {0}, pos = {0};
    if (!count(n, 14) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !as_float(a[11], &eps) || !as_int(a[12], &adjacent)) return NULL;
    const int has_k = a[3] != Py_None;
    if (!look(a[2], "q", &q) || !look(a[4], "q_out", &q_out) || (has_k && (!look(a[3], "k", &k) || !look(a[5], "k_out", &k_out)))) return NULL;
    if (q.ndim != 3 || (q.kind != F16 && q.kind != F32) || q_out.kind != F16 || (has_k && (k.ndim != 3 || k.kind != q.kind || k_out.kind != F16))) {
        refuse("q and k must be [N][heads][D], both fp16 or both fp32, q_out and k_out fp16");
        return NULL;
    }
    const int64_t N = q.size[0], q_heads = q.size[1], kv_heads = has_k ? k.size[1] : 0, D = q.size[2];
    if (!heads(&q, N, q_heads, D, "q", here, &ldq) || !heads(&q_out, N, q_heads, D, "q_out", here, &ldq_out) ||
        (has_k && (!heads(&k, N, kv_heads, D, "k", here, &ldk) || !heads(&k_out, N, kv_heads, D, "k_out", here, &ldk_out))))
        return NULL;
    if (a[7] != Py_None) {
        if (!vector(a[7], F32, "float32", -1, &pairs, "inv_freq", here, &freq) || !look(a[6], "pos", &pos)) return NULL;
        const int last = pos.ndim - 1;
        if (pos.ndim < 1 || pos.ndim > 2 || pos.kind != I32 || pos.device != here || pos.size[last] != N || (N > 1 && pos.step[last] != 1)) {
            refuse("pos must be CUDA int32 [N] or [axes][N] on the current device");
            return NULL;
        }
        axes = pos.ndim == 1 ? 1 : pos.size[0];
        pos_stride = axes <= 1 ? N : pos.step[0];
        if (!sections_of(a[8], axes, pairs, sections)) return NULL;
    }
    if (!vector(a[9], F16, "float16", D, NULL, "q_weight", here, &qw) || !vector(a[10], F16, "float16", D, NULL, "k_weight", here, &kw) ||
        !stream_of(a[13], a[2], here, &stream))
        return NULL;
    if (q_heads > INT32_MAX || kv_heads > INT32_MAX || D > INT32_MAX || pairs > INT32_MAX || axes > INT32_MAX) {
        refuse("heads, their size and the axes must fit 32 bits");
        return NULL;
    }
    Py_BEGIN_ALLOW_THREADS
    st = ((heads_fn)f)(q.p, ldq, k.p, ldk, q.kind == F32, N, (int)q_heads, (int)kv_heads, (int)D, qw, kw, eps, pos.p, pos_stride, (int)axes, freq != NULL ? sections : NULL,
                       freq, (int)pairs, adjacent, q_out.p, ldq_out, k_out.p, ldk_out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* The pages of a cache. */
static int cache_of(PyObject* o, int64_t kv_heads, int64_t dim, int page_tokens, int here, tensor* t) {
    if (!look(o, "cache", t)) return 0;
    if (t->ndim != 2 || t->kind != U8 || t->device != here || !contiguous(t) || t->size[1] != kv_heads * page_tokens * (dim + dim / 8))
        return refuse("cache must be a contiguous CUDA uint8 [pages][spdp_kv4_page_bytes(kv_heads, head_dim, page_tokens)] on the current device");
    return 1;
}

typedef int (*store_fn)(const void*, int64_t, const void*, int64_t, int, int64_t, int, int, const void*, void*, int64_t, int, void*, int64_t, void*, int64_t, void*);
/* the device, k, v, slot, cache, page_tokens, k_values, v_values, stream */
static PyObject* call_kv4_store(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *slot, *stream;
    int64_t ldk, ldv, ldk_values = 0, ldv_values = 0;
    int here, page, st;
    tensor k, v, cache, k_values = {0}, v_values = {0};
    if (!count(n, 10) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !as_int(a[6], &page) || !look(a[2], "k", &k) || !look(a[3], "v", &v) ||
        (a[7] != Py_None && !look(a[7], "k_values", &k_values)) || (a[8] != Py_None && !look(a[8], "v_values", &v_values)))
        return NULL;
    if (k.ndim != 3 || k.kind != F16 || (v.kind != F16 && v.kind != F32) || (a[7] != Py_None && k_values.kind != F16) || (a[8] != Py_None && v_values.kind != F16)) {
        refuse("k must be fp16 [N][kv_heads][D], v fp16 or fp32, k_values and v_values fp16");
        return NULL;
    }
    if (a[4] == Py_None) {
        refuse("slot is required");
        return NULL;
    }
    const int64_t N = k.size[0], kv_heads = k.size[1], D = k.size[2];
    if (!heads(&k, N, kv_heads, D, "k", here, &ldk) || !heads(&v, N, kv_heads, D, "v", here, &ldv) || !cache_of(a[5], kv_heads, D, page, here, &cache) ||
        (a[7] != Py_None && !heads(&k_values, N, kv_heads, D, "k_values", here, &ldk_values)) ||
        (a[8] != Py_None && !heads(&v_values, N, kv_heads, D, "v_values", here, &ldv_values)) || !vector(a[4], I64, "int64", N, NULL, "slot", here, &slot) ||
        !stream_of(a[9], a[2], here, &stream))
        return NULL;
    if (kv_heads > INT32_MAX || D > INT32_MAX) { refuse("heads and their size must fit 32 bits"); return NULL; }
    Py_BEGIN_ALLOW_THREADS
    st = ((store_fn)f)(k.p, ldk, v.p, ldv, v.kind == F32, N, (int)kv_heads, (int)D, slot, cache.p, cache.size[0], page, k_values.p, ldk_values, v_values.p, ldv_values,
                       stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*attn_fn)(const void*, int64_t, int64_t, int, int, int, const void*, int64_t, int, const void*, int64_t, int64_t, const void*, float, float, int64_t,
                       float, void*, int64_t, void*, int64_t, void*);
/* the device, q, cache, page_tokens, kv_heads, table, length, y, scale, cap, window, thr, mask, stream */
static PyObject* call_attn_kv4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *length, *stream;
    int64_t ldq, ldy, table_stride, mask_stride = 0, window;
    int here, page, kv_heads, st;
    float scale, cap, thr;
    tensor q, cache, table, y, mask = {0};
    if (!count(n, 15) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !as_int(a[4], &page) || !as_int(a[5], &kv_heads) || !as_float(a[9], &scale) ||
        !as_float(a[10], &cap) || !as_i64(a[11], &window) || !as_float(a[12], &thr) || !look(a[2], "q", &q) || !look(a[6], "table", &table) || !look(a[8], "y", &y))
        return NULL;
    if (q.ndim != 3 || q.kind != F16 || y.kind != F16) {
        refuse("q must be fp16 [B][q_heads][D] and y fp16");
        return NULL;
    }
    if (table.kind != I32 || table.ndim != 2 || a[7] == Py_None) {
        refuse("table must be int32 [B][pages] and length int32 [B]");
        return NULL;
    }
    const int64_t B = q.size[0], q_heads = q.size[1], D = q.size[2];
    if (!heads(&q, B, q_heads, D, "q", here, &ldq) || !rows(&y, B, q_heads * D, "y", here, &ldy) || !cache_of(a[3], kv_heads, D, page, here, &cache) ||
        !rows(&table, B, table.size[1], "table", here, &table_stride) || !vector(a[7], I32, "int32", B, NULL, "length", here, &length))
        return NULL;
    if (a[13] != Py_None) {
        if (!look(a[13], "mask", &mask)) return NULL;
        if (mask.ndim != 2 || (mask.kind != I32 && mask.kind != U32)) {
            refuse("mask must be 32-bit integers, int32 or uint32 [B][words]");
            return NULL;
        }
        if (!rows(&mask, B, mask.size[1], "mask", here, &mask_stride)) return NULL;
        if (mask.size[1] < q_heads * D / 32) {
            refuse("mask must hold a bit for each column of y");
            return NULL;
        }
    }
    if (!stream_of(a[14], a[2], here, &stream)) return NULL;
    if (q_heads > INT32_MAX || D > INT32_MAX) { refuse("heads and their size must fit 32 bits"); return NULL; }
    Py_BEGIN_ALLOW_THREADS
    st = ((attn_fn)f)(q.p, ldq, B, (int)q_heads, kv_heads, (int)D, cache.p, cache.size[0], page, table.p, table_stride, table.size[1], length, scale, cap, window, thr, y.p, ldy,
                      mask.p, mask_stride, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* The pages of an 8-bit cache. */
static int cache8_of(PyObject* o, int64_t kv_heads, int64_t dim, int page_tokens, int here, tensor* t) {
    if (!look(o, "cache", t)) return 0;
    if (t->ndim != 2 || t->kind != U8 || t->device != here || !contiguous(t) || t->size[1] != kv_heads * page_tokens * (2 * dim + 1))
        return refuse("cache must be a contiguous CUDA uint8 [pages][spdp_kv8_page_bytes(kv_heads, head_dim, page_tokens)] on the current device");
    return 1;
}

/* The requests of N tokens: first [B + 1] or None (a token each), table [B][pages], length [B]. */
typedef struct { void *first, *length; tensor table; int64_t B, stride; } requests;
static int requests_of(PyObject* first, PyObject* table, PyObject* length, int64_t N, int here, requests* r) {
    if (!look(table, "table", &r->table)) return 0;
    if (r->table.kind != I32 || r->table.ndim != 2 || length == Py_None) return refuse("table must be int32 [B][pages] and length int32 [B]");
    r->B = r->table.size[0];
    if (first == Py_None && r->B != N) return refuse("table must have a row for each token where first is None");
    return rows(&r->table, r->B, r->table.size[1], "table", here, &r->stride) && vector(length, I32, "int32", r->B, NULL, "length", here, &r->length) &&
           vector(first, I32, "int32", r->B + 1, NULL, "first", here, &r->first);
}

typedef int (*store8_fn)(const void*, int64_t, const void*, int64_t, int, int64_t, int, int, int64_t, const void*, const void*, int64_t, int64_t, const void*, void*, int64_t,
                         int, void*, int64_t, void*, int64_t, void*);
/* the device, k, v, cache, page_tokens, table, length, first, k_values, v_values, stream */
static PyObject* call_kv8_store(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream;
    int64_t ldk, ldv, ldk_values = 0, ldv_values = 0;
    int here, page, st;
    tensor k, v, cache, k_values = {0}, v_values = {0};
    requests r;
    if (!count(n, 12) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !as_int(a[5], &page) || !look(a[2], "k", &k) || !look(a[3], "v", &v) ||
        (a[9] != Py_None && !look(a[9], "k_values", &k_values)) || (a[10] != Py_None && !look(a[10], "v_values", &v_values)))
        return NULL;
    if (k.ndim != 3 || k.kind != F16 || (v.kind != F16 && v.kind != F32) || (a[9] != Py_None && k_values.kind != F16) || (a[10] != Py_None && v_values.kind != F16)) {
        refuse("k must be fp16 [N][kv_heads][D], v fp16 or fp32, k_values and v_values fp16");
        return NULL;
    }
    const int64_t N = k.size[0], kv_heads = k.size[1], D = k.size[2];
    if (!heads(&k, N, kv_heads, D, "k", here, &ldk) || !heads(&v, N, kv_heads, D, "v", here, &ldv) || !cache8_of(a[4], kv_heads, D, page, here, &cache) ||
        (a[9] != Py_None && !heads(&k_values, N, kv_heads, D, "k_values", here, &ldk_values)) ||
        (a[10] != Py_None && !heads(&v_values, N, kv_heads, D, "v_values", here, &ldv_values)) || !requests_of(a[8], a[6], a[7], N, here, &r) ||
        !stream_of(a[11], a[2], here, &stream))
        return NULL;
    if (kv_heads > INT32_MAX || D > INT32_MAX) { refuse("heads and their size must fit 32 bits"); return NULL; }
    Py_BEGIN_ALLOW_THREADS
    st = ((store8_fn)f)(k.p, ldk, v.p, ldv, v.kind == F32, N, (int)kv_heads, (int)D, r.B, r.first, r.table.p, r.stride, r.table.size[1], r.length, cache.p, cache.size[0], page,
                        k_values.p, ldk_values, v_values.p, ldv_values, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*attn8_fn)(const void*, int64_t, int64_t, int, int, int, int64_t, const void*, const void*, int64_t, int, const void*, int64_t, int64_t, const void*, float, float,
                        int64_t, int64_t, float, void*, int64_t, void*, int64_t, void*);
/* the device, q, cache, page_tokens, kv_heads, table, length, y, scale, first, cap, window, sinks, thr, mask, stream */
static PyObject* call_attn_kv8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream;
    int64_t ldq, ldy, mask_stride = 0, window, sinks;
    int here, page, kv_heads, st;
    float scale, cap, thr;
    tensor q, cache, y, mask = {0};
    requests r;
    if (!count(n, 17) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !as_int(a[4], &page) || !as_int(a[5], &kv_heads) || !as_float(a[9], &scale) ||
        !as_float(a[11], &cap) || !as_i64(a[12], &window) || !as_i64(a[13], &sinks) || !as_float(a[14], &thr) || !look(a[2], "q", &q) || !look(a[8], "y", &y))
        return NULL;
    if (q.ndim != 3 || q.kind != F16 || y.kind != F16) {
        refuse("q must be fp16 [N][q_heads][D] and y fp16");
        return NULL;
    }
    const int64_t N = q.size[0], q_heads = q.size[1], D = q.size[2];
    if (!heads(&q, N, q_heads, D, "q", here, &ldq) || !rows(&y, N, q_heads * D, "y", here, &ldy) || !cache8_of(a[3], kv_heads, D, page, here, &cache) ||
        !requests_of(a[10], a[6], a[7], N, here, &r))
        return NULL;
    if (a[15] != Py_None) {
        if (!look(a[15], "mask", &mask)) return NULL;
        if (mask.ndim != 2 || (mask.kind != I32 && mask.kind != U32)) {
            refuse("mask must be 32-bit integers, int32 or uint32 [N][words]");
            return NULL;
        }
        if (!rows(&mask, N, mask.size[1], "mask", here, &mask_stride)) return NULL;
        if (mask.size[1] < q_heads * D / 32) {
            refuse("mask must hold a bit for each column of y");
            return NULL;
        }
    }
    if (!stream_of(a[16], a[2], here, &stream)) return NULL;
    if (q_heads > INT32_MAX || D > INT32_MAX) { refuse("heads and their size must fit 32 bits"); return NULL; }
    Py_BEGIN_ALLOW_THREADS
    st = ((attn8_fn)f)(q.p, ldq, N, (int)q_heads, kv_heads, (int)D, r.B, r.first, cache.p, cache.size[0], page, r.table.p, r.stride, r.table.size[1], r.length, scale, cap, window,
                       sinks, thr, y.p, ldy, mask.p, mask_stride, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* [pages][bytes] or [layers][pages][bytes], layers apart as they may be. */
static int pages_of(PyObject* o, int here, tensor* t, int* layers, int64_t* stride) {
    if (!look(o, "cache", t)) return 0;
    if (t->ndim == 2) {
        t->size[2] = t->size[1], t->step[2] = t->step[1], t->size[1] = t->size[0], t->step[1] = t->step[0];
        t->size[0] = 1, t->step[0] = t->size[1] * t->size[2], t->ndim = 3;
    }
    if (t->ndim != 3 || t->kind != U8 || t->device != here || (t->size[2] > 1 && t->step[2] != 1) || (t->size[1] > 1 && t->step[1] != t->size[2]) || t->size[0] > INT32_MAX)
        return refuse("cache must be CUDA uint8 [pages][bytes] or [layers][pages][bytes] on the current device, contiguous within a layer");
    *layers = (int)t->size[0], *stride = t->step[0];
    return 1;
}

typedef struct { void *ref, *a, *b, *c, *number; tensor table; int64_t pages, stride, n; } page_lists;
/* ref int32 [pages], table int32 [rows][entries], three int32 [n], an int32 [1] or None */
static int page_lists_of(PyObject* ref, PyObject* table, PyObject* a, PyObject* b, PyObject* c, const char* na, const char* nb, const char* nc, PyObject* number, const char* nn,
                         int here, page_lists* l) {
    l->a = l->b = l->c = NULL, l->n = 0;
    if (ref == Py_None || (a != NULL && (a == Py_None || b == Py_None || c == Py_None))) return refuse("ref and the lists are required");
    if (!look(table, "table", &l->table)) return 0;
    if (l->table.kind != I32 || l->table.ndim != 2) return refuse("table must be int32 [rows][pages of a request]");
    return rows(&l->table, l->table.size[0], l->table.size[1], "table", here, &l->stride) && vector(ref, I32, "int32", -1, &l->pages, "ref", here, &l->ref) &&
           (a == NULL || (vector(a, I32, "int32", -1, &l->n, na, here, &l->a) && vector(b, I32, "int32", l->n, NULL, nb, here, &l->b) &&
                          vector(c, I32, "int32", l->n, NULL, nc, here, &l->c))) &&
           vector(number, I32, "int32", 1, NULL, nn, here, &l->number);
}

typedef int (*take_fn)(void*, int64_t, void*, int64_t, int64_t, int64_t, const void*, const void*, const void*, int64_t, void*, void*);
/* the device, ref, table, row, start, stop, short, stream */
static PyObject* call_kv_pages_take(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream;
    int here, st;
    page_lists l;
    if (!count(n, 9) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !page_lists_of(a[2], a[3], a[4], a[5], a[6], "row", "start", "stop", a[7], "short", here, &l) ||
        !stream_of(a[8], a[2], here, &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((take_fn)f)(l.ref, l.pages, l.table.p, l.table.size[0], l.stride, l.table.size[1], l.a, l.b, l.c, l.n, l.number, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*free_fn)(void*, int64_t, void*, int64_t, int64_t, int64_t, const void*, const void*, const void*, int64_t, void*);
/* the device, ref, table, row, start, stop, stream */
static PyObject* call_kv_pages_free(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream;
    int here, st;
    page_lists l;
    if (!count(n, 8) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !page_lists_of(a[2], a[3], a[4], a[5], a[6], "row", "start", "stop", Py_None, "", here, &l) ||
        !stream_of(a[7], a[2], here, &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((free_fn)f)(l.ref, l.pages, l.table.p, l.table.size[0], l.stride, l.table.size[1], l.a, l.b, l.c, l.n, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* ref has a count for each of the cache's pages */
static int same_pages(const page_lists* l, const tensor* cache) { return l->pages == cache->size[1] || refuse("ref must have a count for each page of the cache"); }

typedef int (*fork_fn)(void*, int, int64_t, int64_t, void*, int64_t, void*, int64_t, int64_t, int64_t, int, const void*, const void*, const void*, int64_t, void*, void*);
/* the device, cache, ref, table, page_tokens, parent, child, length, short, stream */
static PyObject* call_kv_pages_fork(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream;
    int here, st, layers, page;
    int64_t layer_stride;
    tensor cache;
    page_lists l;
    if (!count(n, 11) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !as_int(a[5], &page) || !pages_of(a[2], here, &cache, &layers, &layer_stride) ||
        !page_lists_of(a[3], a[4], a[6], a[7], a[8], "parent", "child", "length", a[9], "short", here, &l) || !same_pages(&l, &cache) || !stream_of(a[10], a[2], here, &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((fork_fn)f)(cache.p, layers, layer_stride, cache.size[2], l.ref, l.pages, l.table.p, l.table.size[0], l.stride, l.table.size[1], page, l.a, l.b, l.c, l.n, l.number, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*copy_fn)(void*, int, int64_t, int64_t, int64_t, const void*, const void*, int64_t, void*);
/* the device, cache, src, dst, stream */
static PyObject* call_kv_pages_copy(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream, *src, *dst;
    int here, st, layers;
    int64_t layer_stride, pairs = 0;
    tensor cache;
    if (!count(n, 6) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !pages_of(a[2], here, &cache, &layers, &layer_stride)) return NULL;
    if (a[3] == Py_None || a[4] == Py_None) { refuse("src and dst are required"); return NULL; }
    if (!vector(a[3], I32, "int32", -1, &pairs, "src", here, &src) || !vector(a[4], I32, "int32", pairs, NULL, "dst", here, &dst) || !stream_of(a[5], a[2], here, &stream)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((copy_fn)f)(cache.p, layers, layer_stride, cache.size[2], cache.size[1], src, dst, pairs, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*compact_fn)(void*, int, int64_t, int64_t, void*, int64_t, void*, int64_t, int64_t, int64_t, void*, void*);
/* the device, cache, ref, table, live, stream */
static PyObject* call_kv_pages_compact(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *stream;
    int here, st, layers;
    int64_t layer_stride;
    tensor cache;
    page_lists l;
    if (!count(n, 7) || !as_ptr(a[0], &f) || !as_int(a[1], &here) || !pages_of(a[2], here, &cache, &layers, &layer_stride) ||
        !page_lists_of(a[3], a[4], NULL, NULL, NULL, "", "", "", a[5], "live", here, &l) || !same_pages(&l, &cache) || !stream_of(a[6], a[2], here, &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((compact_fn)f)(cache.p, layers, layer_stride, cache.size[2], l.ref, l.pages, l.table.p, l.table.size[0], l.stride, l.table.size[1], l.number, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

static PyMethodDef methods[] = {
    {"spmspv", (PyCFunction)(void (*)(void))call_spmspv, METH_FASTCALL, "spdp_spmspv"},
    {"spmspv_batch", (PyCFunction)(void (*)(void))call_spmspv_batch, METH_FASTCALL, "spdp_spmspv_batch"},
    {"spmm", (PyCFunction)(void (*)(void))call_spmm, METH_FASTCALL, "spdp_spmm"},
    {"swiglu_dp", (PyCFunction)(void (*)(void))call_swiglu_dp, METH_FASTCALL, "spdp_swiglu_dp"},
    {"lora", (PyCFunction)(void (*)(void))call_lora, METH_FASTCALL, "spdp_lora"},
    {"qk_norm_rope", (PyCFunction)(void (*)(void))call_qk_norm_rope, METH_FASTCALL, "spdp_qk_norm_rope"},
    {"kv4_store", (PyCFunction)(void (*)(void))call_kv4_store, METH_FASTCALL, "spdp_kv4_store"},
    {"attn_kv4", (PyCFunction)(void (*)(void))call_attn_kv4, METH_FASTCALL, "spdp_attn_kv4"},
    {"kv8_store", (PyCFunction)(void (*)(void))call_kv8_store, METH_FASTCALL, "spdp_kv8_store"},
    {"attn_kv8", (PyCFunction)(void (*)(void))call_attn_kv8, METH_FASTCALL, "spdp_attn_kv8"},
    {"kv_pages_take", (PyCFunction)(void (*)(void))call_kv_pages_take, METH_FASTCALL, "spdp_kv_pages_take"},
    {"kv_pages_free", (PyCFunction)(void (*)(void))call_kv_pages_free, METH_FASTCALL, "spdp_kv_pages_free"},
    {"kv_pages_fork", (PyCFunction)(void (*)(void))call_kv_pages_fork, METH_FASTCALL, "spdp_kv_pages_fork"},
    {"kv_pages_copy", (PyCFunction)(void (*)(void))call_kv_pages_copy, METH_FASTCALL, "spdp_kv_pages_copy"},
    {"kv_pages_compact", (PyCFunction)(void (*)(void))call_kv_pages_compact, METH_FASTCALL, "spdp_kv_pages_compact"},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", "Per-token entry points of libspdp.", -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__pycall(void) { return PyModule_Create(&module); }
