/* The Python side's calls that are made once per layer and token, as vectorcall functions: ctypes converts eight arguments
 * in 1.1 us, a quarter of what such a call costs on the host; this takes 0.2.  Every function gets the address of the
 * library's entry point first (so it follows whichever build of the library is loaded) and then that entry point's arguments
 * as numbers, None for a null pointer.  The status comes back as an int; the GIL is released around the call. */
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

typedef int (*lora_fn)(const void*, int64_t, int64_t, int64_t, const void*, const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, int,
                       const void*, const void*, const void*, int64_t, void*, int64_t, int64_t, int, void*);
static PyObject* call_lora(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *x, *adapter, *wa, *wb, *ranks, *scales, *base, *y, *stream;
    int64_t rows, k, ldx, lda, stride_a, ldb, stride_b, cnt, ldbase, m, ldy;
    int rank, ydt, st;
    if (!count(n, 23) || !as_ptr(a[0], &f) || !as_ptr(a[1], &x) || !as_i64(a[2], &rows) || !as_i64(a[3], &k) || !as_i64(a[4], &ldx) || !as_ptr(a[5], &adapter) ||
        !as_ptr(a[6], &wa) || !as_i64(a[7], &lda) || !as_i64(a[8], &stride_a) || !as_ptr(a[9], &wb) || !as_i64(a[10], &ldb) || !as_i64(a[11], &stride_b) ||
        !as_i64(a[12], &cnt) || !as_int(a[13], &rank) || !as_ptr(a[14], &ranks) || !as_ptr(a[15], &scales) || !as_ptr(a[16], &base) || !as_i64(a[17], &ldbase) ||
        !as_ptr(a[18], &y) || !as_i64(a[19], &m) || !as_i64(a[20], &ldy) || !as_int(a[21], &ydt) || !as_ptr(a[22], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((lora_fn)f)(x, rows, k, ldx, adapter, wa, lda, stride_a, wb, ldb, stride_b, cnt, rank, ranks, scales, base, ldbase, y, m, ldy, ydt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

#define MOST_AXES 4
typedef int (*heads_fn)(const void*, int64_t, const void*, int64_t, int, int64_t, int, int, int, const void*, const void*, float, const void*, int64_t, int,
                        const int*, const void*, int, int, void*, int64_t, void*, int64_t, void*);
/* The sections come as a tuple of ints, one for each axis, or None. */
static PyObject* call_qk_norm_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *q, *k, *qw, *kw, *pos, *freq, *q_out, *k_out, *stream;
    int64_t ldq, ldk, rows, pos_stride, ldq_out, ldk_out;
    int dt, q_heads, kv_heads, dim, axes, pairs, adjacent, st, sections[MOST_AXES] = {0};
    float eps;
    if (!count(n, 25) || !as_ptr(a[0], &f) || !as_ptr(a[1], &q) || !as_i64(a[2], &ldq) || !as_ptr(a[3], &k) || !as_i64(a[4], &ldk) || !as_int(a[5], &dt) ||
        !as_i64(a[6], &rows) || !as_int(a[7], &q_heads) || !as_int(a[8], &kv_heads) || !as_int(a[9], &dim) || !as_ptr(a[10], &qw) || !as_ptr(a[11], &kw) ||
        !as_float(a[12], &eps) || !as_ptr(a[13], &pos) || !as_i64(a[14], &pos_stride) || !as_int(a[15], &axes) || !as_ptr(a[17], &freq) || !as_int(a[18], &pairs) ||
        !as_int(a[19], &adjacent) || !as_ptr(a[20], &q_out) || !as_i64(a[21], &ldq_out) || !as_ptr(a[22], &k_out) || !as_i64(a[23], &ldk_out) || !as_ptr(a[24], &stream))
        return NULL;
    if (a[16] != Py_None) {
        if (!PyTuple_Check(a[16]) || PyTuple_GET_SIZE(a[16]) != axes) {
            PyErr_SetString(PyExc_TypeError, "sections: a tuple of one int for each axis");
            return NULL;
        }
        for (int i = 0; i < axes && i < MOST_AXES; ++i)
            if (!as_int(PyTuple_GET_ITEM(a[16], i), &sections[i])) return NULL;
    }
    Py_BEGIN_ALLOW_THREADS
    st = ((heads_fn)f)(q, ldq, k, ldk, dt, rows, q_heads, kv_heads, dim, qw, kw, eps, pos, pos_stride, axes, a[16] != Py_None ? sections : NULL, freq, pairs, adjacent,
                       q_out, ldq_out, k_out, ldk_out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*store_fn)(const void*, int64_t, const void*, int64_t, int, int64_t, int, int, const void*, void*, int64_t, int, void*, int64_t, void*, int64_t, void*);
static PyObject* call_kv4_store(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *k, *v, *slot, *cache, *k_values, *v_values, *stream;
    int64_t ldk, ldv, rows, pages, ldk_values, ldv_values;
    int vdt, heads, dim, page, st;
    if (!count(n, 18) || !as_ptr(a[0], &f) || !as_ptr(a[1], &k) || !as_i64(a[2], &ldk) || !as_ptr(a[3], &v) || !as_i64(a[4], &ldv) || !as_int(a[5], &vdt) ||
        !as_i64(a[6], &rows) || !as_int(a[7], &heads) || !as_int(a[8], &dim) || !as_ptr(a[9], &slot) || !as_ptr(a[10], &cache) || !as_i64(a[11], &pages) ||
        !as_int(a[12], &page) || !as_ptr(a[13], &k_values) || !as_i64(a[14], &ldk_values) || !as_ptr(a[15], &v_values) || !as_i64(a[16], &ldv_values) ||
        !as_ptr(a[17], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((store_fn)f)(k, ldk, v, ldv, vdt, rows, heads, dim, slot, cache, pages, page, k_values, ldk_values, v_values, ldv_values, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

typedef int (*attn_fn)(const void*, int64_t, int64_t, int, int, int, const void*, int64_t, int, const void*, int64_t, int64_t, const void*, float, float, int64_t,
                       float, void*, int64_t, void*, int64_t, void*);
static PyObject* call_attn_kv4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *f, *q, *cache, *table, *length, *y, *mask, *stream;
    int64_t ldq, batch, pages, table_stride, table_pages, window, ldy, mask_stride;
    int q_heads, kv_heads, dim, page, st;
    float scale, cap, thr;
    if (!count(n, 23) || !as_ptr(a[0], &f) || !as_ptr(a[1], &q) || !as_i64(a[2], &ldq) || !as_i64(a[3], &batch) || !as_int(a[4], &q_heads) || !as_int(a[5], &kv_heads) ||
        !as_int(a[6], &dim) || !as_ptr(a[7], &cache) || !as_i64(a[8], &pages) || !as_int(a[9], &page) || !as_ptr(a[10], &table) || !as_i64(a[11], &table_stride) ||
        !as_i64(a[12], &table_pages) || !as_ptr(a[13], &length) || !as_float(a[14], &scale) || !as_float(a[15], &cap) || !as_i64(a[16], &window) || !as_float(a[17], &thr) ||
        !as_ptr(a[18], &y) || !as_i64(a[19], &ldy) || !as_ptr(a[20], &mask) || !as_i64(a[21], &mask_stride) || !as_ptr(a[22], &stream))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = ((attn_fn)f)(q, ldq, batch, q_heads, kv_heads, dim, cache, pages, page, table, table_stride, table_pages, length, scale, cap, window, thr, y, ldy, mask,
                      mask_stride, stream);
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
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", "Per-token entry points of libspdp.", -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__pycall(void) { return PyModule_Create(&module); }
