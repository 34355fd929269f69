/* CPython entry to the C ABI for the calls a serving loop makes per layer or per token: one METH_FASTCALL function per
 * call, arguments in the order of the header, pointers as integers (None = NULL), the status code returned.  ctypes takes
 * about 4 us to marshal such a call (eighteen arguments), this 0.5 us; the GIL is released meanwhile, as ctypes does. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <string.h>

#include "semanticache.h"

static void* ptr(PyObject* o) { return o == Py_None ? NULL : (void*)PyLong_AsUnsignedLongLong(o); }
/* integers modulo 2^32: what ctypes' c_int32 and c_uint32 take */
static uint32_t u32(PyObject* o) { return (uint32_t)PyLong_AsUnsignedLongMask(o); }
static int32_t i32(PyObject* o) { return (int32_t)u32(o); }
static size_t sz(PyObject* o) { return (size_t)PyLong_AsUnsignedLongLong(o); }
static float f32(PyObject* o) { return (float)PyFloat_AsDouble(o); }

static int arity(Py_ssize_t n, Py_ssize_t want, const char* name) {
    if (n == want) return 1;
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, n);
    return 0;
}
/* anything that has a length and can be iterated, its items made ints; the length, or -1 with an exception set.  One too many
 * is kept: the library refuses the count. */
static int32_t ids_of(PyObject* seq, int32_t* out) {
    if (PyObject_Size(seq) < 0) return -1;
    PyObject* fast = PySequence_Fast(seq, "delim_ids must be a sequence");
    if (!fast) return -1;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
    for (Py_ssize_t i = 0; i < n && i < SC_MAX_DELIMS; ++i) {
        PyObject* v = PyNumber_Long(PySequence_Fast_GET_ITEM(fast, i));
        if (v) { out[i] = i32(v); Py_DECREF(v); }
        if (PyErr_Occurred()) { Py_DECREF(fast); return -1; }
    }
    Py_DECREF(fast);
    return n > SC_MAX_DELIMS ? SC_MAX_DELIMS + 1 : (int32_t)n;
}
#define CALL(expr)                          \
    do {                                    \
        if (PyErr_Occurred()) return NULL;  \
        sc_status code_;                    \
        Py_BEGIN_ALLOW_THREADS              \
        code_ = (expr);                     \
        Py_END_ALLOW_THREADS                \
        return PyLong_FromLong((long)code_);\
    } while (0)

static PyObject* chunk_sizes(PyObject* self, PyObject* const* a, Py_ssize_t n) {   /* B, n -> code, segments, tiles, bytes */
    int32_t segs = 0, tiles = 0;
    (void)self;
    if (!arity(n, 2, "chunk_sizes")) return NULL;
    const int32_t B = i32(a[0]), len = i32(a[1]);
    if (PyErr_Occurred()) return NULL;
    const sc_status code = sc_chunk_bounds(B, len, &segs, &tiles);
    return Py_BuildValue("iiin", (int)code, (int)segs, (int)tiles, (Py_ssize_t)sc_chunk_workspace_bytes(B, len));
}
static PyObject* chunk(PyObject* self, PyObject* const* a, Py_ssize_t n) {   /* delim_ids, n_delim -> one sequence */
    int32_t delims[SC_MAX_DELIMS + 1];
    (void)self;
    if (!arity(n, 16, "chunk")) return NULL;
    const int32_t nd = ids_of(a[3], delims);
    if (nd < 0) return NULL;
    const void* ids = ptr(a[0]);
    const int32_t B = i32(a[1]), len = i32(a[2]), max_len = i32(a[4]), seg_cap = i32(a[6]), tile_cap = i32(a[10]);
    void *seg_off = ptr(a[5]), *seq_off = ptr(a[7]), *n_seg = ptr(a[8]), *tile_seg = ptr(a[9]), *tile_cnt = ptr(a[11]), *ws = ptr(a[12]),
         *status = ptr(a[14]), *stream = ptr(a[15]);
    const size_t bytes = sz(a[13]);
    CALL(sc_chunk(ids, B, len, delims, nd, max_len, seg_off, seg_cap, seq_off, n_seg, tile_seg, tile_cap, tile_cnt, ws, bytes, status, stream));
}
static PyObject* compress(PyObject* self, PyObject* const* a, Py_ssize_t n) {   /* strides and params flattened */
    (void)self;
    if (!arity(n, 28, "compress")) return NULL;
    const void *K = ptr(a[0]), *V = ptr(a[1]);
    const sc_strides st = {PyLong_AsLongLong(a[2]), PyLong_AsLongLong(a[3]), PyLong_AsLongLong(a[4])};
    const sc_dtype dt = (sc_dtype)i32(a[5]);
    const int32_t B = i32(a[6]), H = i32(a[7]), len = i32(a[8]), d = i32(a[9]), tile_cap = i32(a[15]), cap = i32(a[22]);
    const void *seg_off = ptr(a[10]), *seq_off = ptr(a[11]), *n_seg = ptr(a[12]), *tile_seg = ptr(a[13]), *tile_cnt = ptr(a[14]);
    const sc_gsc_params prm = {f32(a[16]), i32(a[17]), u32(a[18])};
    void *core_k = ptr(a[19]), *core_v = ptr(a[20]), *count = ptr(a[21]), *core_len = ptr(a[23]), *assign = ptr(a[24]), *ws = ptr(a[25]);
    const size_t bytes = sz(a[26]);
    PyObject* tail = a[27];   /* (status, stream) */
    if (!PyTuple_Check(tail) || PyTuple_GET_SIZE(tail) != 2) { PyErr_SetString(PyExc_TypeError, "(status, stream) expected"); return NULL; }
    void *status = ptr(PyTuple_GET_ITEM(tail, 0)), *stream = ptr(PyTuple_GET_ITEM(tail, 1));
    CALL(sc_compress(K, V, st, dt, B, H, len, d, seg_off, seq_off, n_seg, tile_seg, tile_cnt, tile_cap, &prm, core_k, core_v, count, cap,
                     core_len, assign, ws, bytes, status, stream));
}
static PyObject* decode_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    if (!arity(n, 18, "decode_attn")) return NULL;
    const void *q = ptr(a[0]), *core_k = ptr(a[6]), *core_v = ptr(a[7]), *count = ptr(a[8]), *core_len = ptr(a[10]);
    const sc_dtype dt = (sc_dtype)i32(a[1]);
    const int32_t B = i32(a[2]), Hq = i32(a[3]), Hkv = i32(a[4]), d = i32(a[5]), cap = i32(a[9]);
    const float scale = f32(a[11]);
    const uint32_t flags = u32(a[12]);
    void *out = ptr(a[13]), *ws = ptr(a[14]), *status = ptr(a[16]), *stream = ptr(a[17]);
    const size_t bytes = sz(a[15]);
    CALL(sc_decode_attn(q, dt, B, Hq, Hkv, d, core_k, core_v, count, cap, core_len, scale, flags, out, ws, bytes, status, stream));
}
static PyObject* prefill_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    if (!arity(n, 17, "prefill_attn")) return NULL;
    const void *q = ptr(a[0]), *core_k = ptr(a[7]), *core_v = ptr(a[8]), *count = ptr(a[9]), *core_len = ptr(a[11]);
    const sc_dtype dt = (sc_dtype)i32(a[1]);
    const int32_t B = i32(a[2]), Hq = i32(a[3]), Hkv = i32(a[4]), m = i32(a[5]), d = i32(a[6]), cap = i32(a[10]);
    const float scale = f32(a[12]);
    const uint32_t flags = u32(a[13]);
    void *out = ptr(a[14]), *status = ptr(a[15]), *stream = ptr(a[16]);
    CALL(sc_prefill_attn(q, dt, B, Hq, Hkv, m, d, core_k, core_v, count, cap, core_len, scale, flags, out, status, stream));
}
static PyObject* append(PyObject* self, PyObject* const* a, Py_ssize_t n) {   /* delim_ids, n_delim -> one sequence */
    int32_t delims[SC_MAX_DELIMS + 1];
    (void)self;
    if (!arity(n, 19, "append")) return NULL;
    const int32_t nd = ids_of(a[7], delims);
    if (nd < 0) return NULL;
    const void *k = ptr(a[0]), *v = ptr(a[1]), *ids = ptr(a[6]);
    const sc_dtype dt = (sc_dtype)i32(a[2]);
    const int32_t B = i32(a[3]), H = i32(a[4]), d = i32(a[5]), max_len = i32(a[8]), cap = i32(a[13]);
    const float tau = f32(a[9]);
    void *core_k = ptr(a[10]), *core_v = ptr(a[11]), *count = ptr(a[12]), *core_len = ptr(a[14]), *tail_len = ptr(a[15]),
         *attn_len = ptr(a[16]), *status = ptr(a[17]), *stream = ptr(a[18]);
    CALL(sc_append(k, v, dt, B, H, d, ids, delims, nd, max_len, tau, core_k, core_v, count, cap, core_len, tail_len, attn_len, status, stream));
}
static PyObject* append_layers(PyObject* self, PyObject* const* a, Py_ssize_t n) {   /* delim_ids, n_delim -> one sequence */
    int32_t delims[SC_MAX_DELIMS + 1];
    (void)self;
    if (!arity(n, 13, "append_layers")) return NULL;
    const int32_t nd = ids_of(a[7], delims);
    if (nd < 0) return NULL;
    const void *table = ptr(a[0]), *ids = ptr(a[6]);
    const sc_dtype dt = (sc_dtype)i32(a[2]);
    const int32_t L = i32(a[1]), B = i32(a[3]), H = i32(a[4]), d = i32(a[5]), max_len = i32(a[8]), cap = i32(a[10]);
    const float tau = f32(a[9]);
    void *status = ptr(a[11]), *stream = ptr(a[12]);
    CALL(sc_append_layers(table, L, dt, B, H, d, ids, delims, nd, max_len, tau, cap, status, stream));
}

/* a cache in pages: its six addresses, and the bytes of an sc_paged_cache that has everything but them */
static int cache_of(PyObject* const* a, sc_paged_cache* c) {
    char* form;
    Py_ssize_t n;
    if (PyBytes_AsStringAndSize(a[6], &form, &n) < 0) return 0;
    if (n != (Py_ssize_t)sizeof *c) { PyErr_SetString(PyExc_ValueError, "not the form of a paged cache"); return 0; }
    memcpy(c, form, sizeof *c);
    c->k = ptr(a[0]); c->v = ptr(a[1]); c->table = ptr(a[2]); c->count = ptr(a[3]); c->k_min = ptr(a[4]); c->k_max = ptr(a[5]);
    return 1;
}
/* The calls on a paged cache take the tensors themselves and check them here: what a tensor is asked for from Python costs twice as
 * much, and an append asks eleven of them (4 us of 7.5). */
static PyObject *s_shape, *s_stride, *s_dtype, *s_get_device, *s_data_ptr, *s_numel, *s_is_contiguous, *s_nbytes;
static PyObject *t_int32, *t_float32;   /* the types, from set_types */

static PyObject* set_types(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    if (!arity(n, 2, "set_types")) return NULL;
    Py_INCREF(a[0]); Py_XSETREF(t_int32, a[0]);
    Py_INCREF(a[1]); Py_XSETREF(t_float32, a[1]);
    Py_RETURN_NONE;
}
static int refuse(const char* what, const char* why) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: %s", what, why);
    return 0;
}
static int is_type(PyObject* t, PyObject* type) {
    PyObject* x = PyObject_GetAttr(t, s_dtype);
    Py_XDECREF(x);
    return x != NULL && x == type;
}
static long long asked(PyObject* t, PyObject* method) {   /* of a method that gives an integer; -1 with an exception set */
    PyObject* x = PyObject_CallMethodNoArgs(t, method);
    if (!x) return -1;
    const long long v = PyLong_AsLongLong(x);
    Py_DECREF(x);
    return v;
}
static void* address(PyObject* t) {                       /* None: NULL */
    if (t == Py_None) return NULL;
    PyObject* x = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!x) return NULL;
    void* p = (void*)PyLong_AsUnsignedLongLong(x);
    Py_DECREF(x);
    return p;
}
static int three(PyObject* x, int64_t* v) {               /* a tuple of three integers; the reference is taken */
    if (!x) return 0;
    int ok = PyTuple_Check(x) && PyTuple_GET_SIZE(x) == 3;
    for (int i = 0; ok && i < 3; ++i) {
        v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(x, i));
        if (v[i] == -1 && PyErr_Occurred()) ok = 0;
    }
    Py_DECREF(x);
    return ok;
}
/* rows [n, heads, d]: sizes, element strides (0 where there is one entry) and address */
typedef struct { int64_t n, heads, s0, s1; void* at; } rows3;
static int rows_of(PyObject* t, PyObject* type, long dev, int64_t d, rows3* r, const char* what) {
    int64_t size[3], step[3];
    if (!is_type(t, type)) return refuse(what, "not of the cache's type");
    if (asked(t, s_get_device) != dev) return refuse(what, "not on the cache's device");
    if (!three(PyObject_GetAttr(t, s_shape), size) || !three(PyObject_CallMethodNoArgs(t, s_stride), step)) return refuse(what, "three axes expected");
    if (size[2] != d || (step[2] != 1 && size[0] * size[1] > 0)) return refuse(what, "the last axis is the cache's head dimension, contiguous");
    r->n = size[0]; r->heads = size[1];
    r->s0 = size[0] > 1 ? step[0] : 0; r->s1 = size[1] > 1 ? step[1] : 0;
    r->at = address(t);
    return !PyErr_Occurred();
}
static int solid(const rows3* r, int64_t d) { return (r->n <= 1 || r->s0 == r->heads * d) && (r->heads <= 1 || r->s1 == d); }
/* n contiguous values of a type; None gives NULL */
static int list_of(PyObject* t, PyObject* type, long dev, int64_t n, void** at, const char* what) {
    *at = NULL;
    if (t == Py_None) return 1;
    if (!is_type(t, type)) return refuse(what, "of another type");
    if (asked(t, s_numel) != n) return refuse(what, "of another length");
    if (asked(t, s_get_device) != dev) return refuse(what, "not on the cache's device");
    PyObject* c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    Py_XDECREF(c);
    if (c != Py_True) return refuse(what, "not contiguous");
    *at = address(t);
    return !PyErr_Occurred();
}
/* where the device's errors go: int32, at least one, or None */
static int status_of(PyObject* t, long dev, void** at) {
    *at = NULL;
    if (t == Py_None) return 1;
    if (!is_type(t, t_int32) || asked(t, s_get_device) != dev || asked(t, s_numel) < 1) return refuse("status", "int32 on the cache's device expected");
    *at = address(t);
    return !PyErr_Occurred();
}
/* after the cache: its type's object and number, its device, tables, heads and head dimension */
typedef struct { PyObject* type; sc_dtype dt; long dev; int32_t B, heads, d; } about;
static int about_of(PyObject* const* a, about* c) {
    c->type = a[0]; c->dt = (sc_dtype)i32(a[1]); c->dev = PyLong_AsLong(a[2]); c->B = i32(a[3]); c->heads = i32(a[4]); c->d = i32(a[5]);
    return !PyErr_Occurred();
}
static PyObject* paged_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    sc_paged_cache c;
    sc_paged_rows r;
    about w;
    rows3 k, v, q = {0, 0, 0, 0, NULL}, qo = {0, 0, 0, 0, NULL};
    void *count, *off, *len, *have, *out, *freq, *pos;
    (void)self;
    if (!arity(n, 27, "paged_append") || !cache_of(a, &c) || !about_of(a + 7, &w)) return NULL;
    PyObject* const* t = a + 13;   /* k_new, v_new, seq_off, cache_len, seq_len, count_new, len_out, q, q_out, inv_freq, positions */
    if (!rows_of(t[0], w.type, w.dev, w.d, &k, "k_new") || !rows_of(t[1], w.type, w.dev, w.d, &v, "v_new")) return NULL;
    if (k.n != v.n || k.heads != v.heads || k.s0 != v.s0 || k.s1 != v.s1) { refuse("k_new and v_new", "one shape and layout expected"); return NULL; }
    if (k.heads != w.heads || k.n > INT32_MAX) { refuse("k_new", "as many heads as a page of the cache expected"); return NULL; }
    if (t[2] == Py_None || t[3] == Py_None) { refuse("seq_off, cache_len", "expected"); return NULL; }
    if (!list_of(t[2], t_int32, w.dev, (int64_t)w.B + 1, &off, "seq_off") || !list_of(t[3], t_int32, w.dev, w.B, &have, "cache_len") ||
        !list_of(t[4], t_int32, w.dev, w.B, &len, "seq_len") || !list_of(t[5], t_int32, w.dev, k.n * k.heads, &count, "count_new") ||
        !list_of(t[6], t_int32, w.dev, w.B, &out, "len_out") || !list_of(t[10], t_int32, w.dev, k.n, &pos, "positions")) return NULL;
    if ((t[7] == Py_None) != (t[8] == Py_None)) { refuse("q and q_out", "both or neither expected"); return NULL; }
    if (t[7] != Py_None) {
        if (!rows_of(t[7], w.type, w.dev, w.d, &q, "q") || !rows_of(t[8], w.type, w.dev, w.d, &qo, "q_out")) return NULL;
        if (q.n != k.n || qo.n != k.n || q.heads != qo.heads || q.heads > INT32_MAX) { refuse("q and q_out", "[T, Hq, d] expected"); return NULL; }
    }
    const long long freqs = t[9] == Py_None ? 0 : asked(t[9], s_numel);
    if (PyErr_Occurred() || !list_of(t[9], t_float32, w.dev, freqs, &freq, "inv_freq")) return NULL;
    if (freqs > INT32_MAX / 2) { refuse("inv_freq", "too long"); return NULL; }
    r.k = k.at; r.v = v.at; r.kv_token = k.s0; r.kv_head = k.s1; r.count = count; r.seq_off = off; r.seq_len = len; r.cache_len = have; r.len_out = out;
    r.q = q.at; r.q_out = qo.at; r.q_token = q.s0; r.q_head = q.s1; r.qo_token = qo.s0; r.qo_head = qo.s1;
    r.inv_freq = freq; r.rot_dim = 2 * (int32_t)freqs; r.positions = pos;
    const int32_t Hq = r.q != NULL ? (int32_t)q.heads : w.heads, T = (int32_t)k.n;
    const uint32_t flags = u32(a[25]);
    void *status, *stream = ptr(a[26]);
    if (!status_of(a[24], w.dev, &status)) return NULL;
    CALL(sc_paged_append(&c, &r, w.dt, w.B, Hq, w.heads, T, w.d, flags, status, stream));
}
static int query_of(PyObject* t, const about* w, rows3* q, const char* what) {
    if (!rows_of(t, w->type, w->dev, w->d, q, what)) return 0;
    if (q->n != w->B || q->heads > INT32_MAX || !solid(q, w->d)) return refuse(what, "contiguous [B, Hq, d] expected, B as the cache's tables");
    return 1;
}
static PyObject* paged_decode_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {   /* heads: the KV heads; then tables per sequence */
    sc_paged_cache c;
    about w;
    rows3 q, out;
    void* lens;
    (void)self;
    if (!arity(n, 21, "paged_decode_attn") || !cache_of(a, &c) || !about_of(a + 7, &w)) return NULL;
    PyObject* const* t = a + 13;   /* q, lens, out, workspace, scale, status, flags, stream */
    if (!query_of(t[0], &w, &q, "q") || !query_of(t[2], &w, &out, "out")) return NULL;
    if (q.heads != out.heads) { refuse("out", "the shape of q expected"); return NULL; }
    if (t[1] == Py_None || !list_of(t[1], t_int32, w.dev, (int64_t)w.B * c.table_heads, &lens, "lens")) { refuse("lens", "expected"); return NULL; }
    if (t[3] == Py_None || asked(t[3], s_get_device) != w.dev) { refuse("workspace", "expected on the cache's device"); return NULL; }
    PyObject* whole = PyObject_CallMethodNoArgs(t[3], s_is_contiguous);
    Py_XDECREF(whole);
    if (whole != Py_True) { refuse("workspace", "not contiguous"); return NULL; }
    PyObject* bytes = PyObject_GetAttr(t[3], s_nbytes);
    if (!bytes) return NULL;
    const size_t have = sz(bytes);
    Py_DECREF(bytes);
    void *ws = address(t[3]), *status, *stream = ptr(t[7]);
    if (!status_of(t[5], w.dev, &status)) return NULL;
    const float scale = f32(t[4]);
    const uint32_t flags = u32(t[6]);
    CALL(sc_paged_decode_attn(&c, q.at, w.dt, w.B, (int32_t)q.heads, w.heads, w.d, lens, scale, flags, out.at, ws, have, status, stream));
}
static PyObject* paged_select(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    sc_paged_cache c;
    about w;
    rows3 q;
    void *lens, *table, *len;
    (void)self;
    if (!arity(n, 22, "paged_select") || !cache_of(a, &c) || !about_of(a + 7, &w)) return NULL;
    PyObject* const* t = a + 13;   /* q, lens, keep, n_first, n_last, sel_table, sel_len, status, stream */
    const int32_t keep = i32(t[2]), first = i32(t[3]), last = i32(t[4]);
    if (PyErr_Occurred() || !query_of(t[0], &w, &q, "q")) return NULL;
    if (t[1] == Py_None || t[5] == Py_None || t[6] == Py_None) { refuse("lens, sel_table, sel_len", "expected"); return NULL; }
    if (!list_of(t[1], t_int32, w.dev, (int64_t)w.B * c.table_heads, &lens, "lens") ||
        !list_of(t[5], t_int32, w.dev, (int64_t)w.B * w.heads * keep, &table, "sel_table") ||
        !list_of(t[6], t_int32, w.dev, (int64_t)w.B * w.heads, &len, "sel_len")) return NULL;
    void *status, *stream = ptr(t[8]);
    if (!status_of(t[7], w.dev, &status)) return NULL;
    CALL(sc_paged_select(&c, q.at, w.dt, w.B, (int32_t)q.heads, w.heads, w.d, lens, keep, first, last, table, len, status, stream));
}

#define FN(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {FN(chunk_sizes), FN(chunk), FN(compress), FN(decode_attn), FN(prefill_attn), FN(append), FN(append_layers),
                                FN(set_types), FN(paged_append), FN(paged_decode_attn), FN(paged_select), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__native_calls(void) {
    if (!(s_shape = PyUnicode_InternFromString("shape")) || !(s_stride = PyUnicode_InternFromString("stride")) ||
        !(s_dtype = PyUnicode_InternFromString("dtype")) || !(s_get_device = PyUnicode_InternFromString("get_device")) ||
        !(s_data_ptr = PyUnicode_InternFromString("data_ptr")) || !(s_numel = PyUnicode_InternFromString("numel")) ||
        !(s_is_contiguous = PyUnicode_InternFromString("is_contiguous")) || !(s_nbytes = PyUnicode_InternFromString("nbytes"))) return NULL;
    return PyModule_Create(&module);
}
