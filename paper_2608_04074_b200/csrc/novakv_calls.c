/* Python entry to the per-step calls of libnovakv.so: takes tensors, forms the C arguments and calls the library without
 * the interpreter lock.
 *
 * A decode step of one short sequence runs 17 us on the device; marshalled through ctypes, its two calls took the host 27 us
 * (7 us a call for the foreign-function layer, another 2 for the stream object).  Nothing is computed or kept here.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <limits.h>
#include <stdint.h>

#include "novakv.h"

/* How a C argument is formed from Python argument `arg` (the context handle comes first and is not listed):
 *   L an integer   I int(x)   F float(x)   P data_ptr() of a tensor, 0 for None   0, 1 shape[0], shape[1]   n, m the same, 0 for None
 *   T 1 if its dtype is float32   B its size in bytes   S the current CUDA stream (no argument) */
typedef struct { char kind; signed char arg; } param;
#define MAX_ARGS 28

enum { ENCODE, ENCODE_SCALED, ENCODE_DEPLOYED, DECODE, DECODE_SCALED, DECODE_SINK, DECODE_BANDED, DECODE_DEPLOYED, BAND_APPEND,
       WINDOW, STEP_HOST, STEP_HOST_ASYNC, N_ENTRIES };

static const struct { const char* name; int n_args; param p[MAX_ARGS]; } entries[N_ENTRIES] = {
    /* layer, k_new, v_new, tok_seq, tok_pos, k_pages, v_pages, page_table, seq_lens */
    [ENCODE] = {"novakv_encode_append", 9,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'n', 1}, {'P', 5}, {'P', 6}, {'0', 5}, {'P', 7}, {'1', 7}, {'0', 7}, {'P', 8}, {'S', 0}}},
    /* ... k_pages, v_pages, k_scales, page_table, seq_lens */
    [ENCODE_SCALED] = {"novakv_encode_append_scaled", 10,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'n', 1}, {'P', 5}, {'P', 6}, {'P', 7}, {'0', 5}, {'P', 8}, {'1', 8}, {'0', 8}, {'P', 9}, {'S', 0}}},
    /* ... k_pages, v_pages, k_scales, v_meta, page_table, seq_lens */
    [ENCODE_DEPLOYED] = {"novakv_encode_append_deployed", 11,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'n', 1}, {'P', 5}, {'P', 6}, {'P', 7}, {'P', 8}, {'0', 5}, {'P', 9}, {'1', 9}, {'0', 9}, {'P', 10}, {'S', 0}}},
    /* layer, q, k_pages, v_pages, page_table, seq_lens, out, workspace, sm_scale */
    [DECODE] = {"novakv_decode_attention", 9,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'0', 2}, {'P', 4}, {'1', 4}, {'P', 5}, {'0', 1}, {'F', 8}, {'P', 6}, {'T', 6}, {'P', 7}, {'B', 7}, {'S', 0}}},
    /* layer, q, k_pages, v_pages, k_scales, page_table, seq_lens, out, workspace, sm_scale */
    [DECODE_SCALED] = {"novakv_decode_attention_scaled", 10,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'0', 2}, {'P', 5}, {'1', 5}, {'P', 6}, {'0', 1}, {'F', 9}, {'P', 7}, {'T', 7}, {'P', 8}, {'B', 8}, {'S', 0}}},
    /* layer, q, k_pages, v_pages, k_scales, sink_logits, page_table, seq_lens, out, workspace, sm_scale */
    [DECODE_SINK] = {"novakv_decode_attention_sink", 11,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'P', 5}, {'0', 2}, {'P', 6}, {'1', 6}, {'P', 7}, {'0', 1}, {'F', 10}, {'P', 8}, {'T', 8}, {'P', 9}, {'B', 9}, {'S', 0}}},
    /* layer, q, k_pages, v_pages, k_scales, sink_logits, page_table, quant_lens, band_k, band_v, n_sink, band_meta, out, workspace, sm_scale */
    [DECODE_BANDED] = {"novakv_decode_attention_banded", 15,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'P', 5}, {'0', 2}, {'P', 6}, {'1', 6}, {'P', 7}, {'P', 8}, {'P', 9}, {'1', 8}, {'I', 10}, {'P', 11},
         {'0', 1}, {'F', 14}, {'P', 12}, {'T', 12}, {'P', 13}, {'B', 13}, {'S', 0}}},
    /* layer, q, k_pages, v_pages, k_scales, v_meta, sink_logits, page_table, quant_lens, band_k, band_v, n_sink, band_meta, out, workspace, sm_scale */
    [DECODE_DEPLOYED] = {"novakv_decode_attention_deployed", 16,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'P', 5}, {'P', 6}, {'0', 2}, {'P', 7}, {'1', 7}, {'P', 8}, {'P', 9}, {'P', 10}, {'m', 9}, {'I', 11}, {'P', 12},
         {'0', 1}, {'F', 15}, {'P', 13}, {'T', 13}, {'P', 14}, {'B', 14}, {'S', 0}}},
    /* layer, k_new, v_new, band_k, band_v, n_sink, n_rec, block, band_meta, quant_lens, k_pages, v_pages, k_scales, v_meta, page_table, seq_lens, staging */
    [BAND_APPEND] = {"novakv_band_append", 17,
        {{'L', 0}, {'P', 1}, {'P', 2}, {'0', 1}, {'P', 3}, {'P', 4}, {'1', 3}, {'I', 5}, {'I', 6}, {'I', 7}, {'P', 8}, {'P', 9}, {'P', 10}, {'P', 11}, {'P', 12}, {'P', 13},
         {'0', 10}, {'P', 14}, {'1', 14}, {'P', 15}, {'P', 16}, {'B', 16}, {'S', 0}}},
    /* q, k_pages, v_pages, page_table, seq_lens, out, workspace, sm_scale, window */
    [WINDOW] = {"novakv_bf16_decode_attention", 9,
        {{'P', 0}, {'P', 1}, {'P', 2}, {'0', 1}, {'P', 3}, {'1', 3}, {'P', 4}, {'0', 0}, {'F', 7}, {'I', 8}, {'P', 5}, {'T', 5}, {'P', 6}, {'B', 6}, {'S', 0}}},
    /* layer, k_new, v_new, tok_seq, tok_pos, q, k_pages, v_pages, page_table, seq_lens, out, staging, workspace, sm_scale */
#define HOST_PARAMS {{'L', 0}, {'P', 1}, {'P', 2}, {'P', 3}, {'P', 4}, {'n', 1}, {'P', 5}, {'P', 6}, {'P', 7}, {'0', 6}, {'P', 8}, {'1', 8}, {'P', 9}, {'0', 5}, {'F', 13}, \
         {'P', 10}, {'P', 11}, {'B', 11}, {'P', 12}, {'B', 12}, {'S', 0}}
    [STEP_HOST] = {"novakv_step_host", 14, HOST_PARAMS},
    [STEP_HOST_ASYNC] = {"novakv_step_host_async", 14, HOST_PARAMS},
};

static PyObject *s_data_ptr, *s_shape, *s_dtype, *s_nbytes, *s_stride, *s_get_device, *s_is_contiguous;
static PyObject *get_stream, *get_device, *float32;        /* given by setup() */

typedef struct {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    int entry;
    void* fn;
} Entry;

/* shape[dim] as int(x.shape[dim]) gives it; -1 with an exception set */
static long long shape_of(PyObject* x, int dim) {
    PyObject* shape = PyObject_GetAttr(x, s_shape);
    if (!shape) return -1;
    PyObject* item = PySequence_GetItem(shape, dim);
    Py_DECREF(shape);
    if (!item) return -1;
    const long long v = PyLong_AsLongLong(item);
    Py_DECREF(item);
    return v;
}
static int as_int(PyObject* x, int exact, long long* v) {
    PyObject* n = exact ? PyNumber_Index(x) : PyNumber_Long(x);
    if (!n) return -1;
    *v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    return *v == -1 && PyErr_Occurred() ? -1 : 0;
}
static int pointer_of(PyObject* x, unsigned long long* v) {
    if (x == Py_None) { *v = 0; return 0; }
    PyObject* n = PyObject_CallMethodNoArgs(x, s_data_ptr);
    if (!n) return -1;
    *v = PyLong_AsUnsignedLongLong(n);
    Py_DECREF(n);
    return PyErr_Occurred() ? -1 : 0;
}
static int current_stream(unsigned long long* v) {
    PyObject* dev = PyObject_CallNoArgs(get_device);
    if (!dev) return -1;
    PyObject* s = PyObject_CallOneArg(get_stream, dev);
    Py_DECREF(dev);
    if (!s) return -1;
    *v = PyLong_AsUnsignedLongLong(s);
    Py_DECREF(s);
    return PyErr_Occurred() ? -1 : 0;
}

static novakv_status call(int entry, void* fn, novakv_ctx* c, const long long* a, float f) {
#define I(i) ((int)a[i])
#define V(i) ((void*)(uintptr_t)a[i])
#define Z(i) ((size_t)a[i])
    switch (entry) {
        case ENCODE:
            return ((__typeof__(&novakv_encode_append))fn)(c, I(0), V(1), V(2), V(3), V(4), I(5), V(6), V(7), I(8), V(9), I(10), I(11), V(12), V(13));
        case ENCODE_SCALED:
            return ((__typeof__(&novakv_encode_append_scaled))fn)(c, I(0), V(1), V(2), V(3), V(4), I(5), V(6), V(7), V(8), I(9), V(10), I(11), I(12), V(13), V(14));
        case ENCODE_DEPLOYED:
            return ((__typeof__(&novakv_encode_append_deployed))fn)(c, I(0), V(1), V(2), V(3), V(4), I(5), V(6), V(7), V(8), V(9), I(10), V(11), I(12), I(13), V(14), V(15));
        case DECODE:
            return ((__typeof__(&novakv_decode_attention))fn)(c, I(0), V(1), V(2), V(3), I(4), V(5), I(6), V(7), I(8), f, V(10), I(11), V(12), Z(13), V(14));
        case DECODE_SCALED:
            return ((__typeof__(&novakv_decode_attention_scaled))fn)(c, I(0), V(1), V(2), V(3), V(4), I(5), V(6), I(7), V(8), I(9), f, V(11), I(12), V(13), Z(14), V(15));
        case DECODE_SINK:
            return ((__typeof__(&novakv_decode_attention_sink))fn)(c, I(0), V(1), V(2), V(3), V(4), V(5), I(6), V(7), I(8), V(9), I(10), f, V(12), I(13), V(14), Z(15), V(16));
        case DECODE_BANDED:
            return ((__typeof__(&novakv_decode_attention_banded))fn)(c, I(0), V(1), V(2), V(3), V(4), V(5), I(6), V(7), I(8), V(9), V(10), V(11), I(12), I(13), V(14), I(15), f,
                                                                     V(17), I(18), V(19), Z(20), V(21));
        case DECODE_DEPLOYED:
            return ((__typeof__(&novakv_decode_attention_deployed))fn)(c, I(0), V(1), V(2), V(3), V(4), V(5), V(6), I(7), V(8), I(9), V(10), V(11), V(12), I(13), I(14), V(15),
                                                                       I(16), f, V(18), I(19), V(20), Z(21), V(22));
        case BAND_APPEND:
            return ((__typeof__(&novakv_band_append))fn)(c, I(0), V(1), V(2), I(3), V(4), V(5), I(6), I(7), I(8), I(9), V(10), V(11), V(12), V(13), V(14), V(15), I(16), V(17),
                                                         I(18), V(19), V(20), Z(21), V(22));
        case WINDOW:
            return ((__typeof__(&novakv_bf16_decode_attention))fn)(c, V(0), V(1), V(2), I(3), V(4), I(5), V(6), I(7), f, I(9), V(10), I(11), V(12), Z(13), V(14));
        default:
            return ((__typeof__(&novakv_step_host))fn)(c, I(0), V(1), V(2), V(3), V(4), I(5), V(6), V(7), V(8), I(9), V(10), I(11), V(12), I(13), f, V(15), V(16), Z(17), V(18),
                                                       Z(19), V(20));
    }
#undef I
#undef V
#undef Z
}

/* entry(handle, arguments...) -> status */
static PyObject* entry_call(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* kwnames) {
    Entry* e = (Entry*)self;
    const Py_ssize_t n = PyVectorcall_NARGS(nargsf);
    if (kwnames || n != entries[e->entry].n_args + 1) {
        PyErr_Format(PyExc_TypeError, "%s: a context and %d positional arguments", entries[e->entry].name, entries[e->entry].n_args);
        return NULL;
    }
    const unsigned long long ctx = args[0] == Py_None ? 0 : PyLong_AsUnsignedLongLong(args[0]);
    if (PyErr_Occurred()) return NULL;
    long long a[MAX_ARGS];
    float f = 0.f;
    const param* p = entries[e->entry].p;
    for (int i = 0; i < MAX_ARGS && p[i].kind; ++i) {
        PyObject* x = args[1 + p[i].arg];
        unsigned long long u = 0;
        a[i] = 0;
        switch (p[i].kind) {
            case 'L': if (as_int(x, 1, &a[i])) return NULL; break;
            case 'I': if (as_int(x, 0, &a[i])) return NULL; break;
            case 'F': f = (float)PyFloat_AsDouble(x); break;
            case 'P': if (pointer_of(x, &u)) return NULL; a[i] = (long long)u; break;
            case '0': a[i] = shape_of(x, 0); break;
            case '1': a[i] = shape_of(x, 1); break;
            case 'n': if (x != Py_None) a[i] = shape_of(x, 0); break;
            case 'm': if (x != Py_None) a[i] = shape_of(x, 1); break;
            case 'T': { PyObject* d = PyObject_GetAttr(x, s_dtype); a[i] = d == float32; Py_XDECREF(d); break; }
            case 'B': { PyObject* b = PyObject_GetAttr(x, s_nbytes); if (!b) return NULL; a[i] = PyLong_AsLongLong(b); Py_DECREF(b); break; }
            default: if (current_stream(&u)) return NULL; a[i] = (long long)u;
        }
        if (PyErr_Occurred()) return NULL;
    }
    novakv_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call(e->entry, e->fn, (novakv_ctx*)(uintptr_t)ctx, a, f);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

static PyTypeObject EntryType = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "_novakv_calls.Entry",
    .tp_basicsize = sizeof(Entry),
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL,
    .tp_vectorcall_offset = offsetof(Entry, vectorcall),
    .tp_call = PyVectorcall_Call,
};

/* ---- calls around the BF16 and the 4-bit cache: these also check what they are given, before an address goes to a kernel --------
 *
 * How a C argument is formed from Python argument `arg`, and what is asked of it (all tensors on the context's device):
 *   q, k rows [n][Hq or Hkv][d] in bfloat16, heads of a token contiguous; Q, K the same or None   s stride(0) of rows, 0 for None
 *   e output rows [n][Hkv][d], o [n][Hq][d], bfloat16 or float32, contiguous     i [n] int32     t page table int32, two dimensions
 *   l lengths int32, as many as the page table has rows    f float32 [Hq] or None      b, c pool of the BF16, of the 4-bit cache
 *   h transform, an object with data_ptr(); H the same or None    w workspace    N n   0, 1, I, F, T, B, S as above (S of the device) */
enum { QK_NORM_ROPE, BF16_APPEND, INT4_APPEND, INT4_GATHER, INT4_DECODE, N_OPERATORS };
#define APPEND_PARAMS(pool) {{'H', 0}, {'k', 1}, {'s', 1}, {'k', 2}, {'s', 2}, {'i', 3}, {'i', 4}, {'N', 0}, {pool, 5}, {pool, 6}, {'0', 5}, {'t', 7}, {'1', 7}, {'0', 7}, \
         {'l', 8}, {'Q', 9}, {'s', 9}, {'Q', 10}, {'s', 10}, {'S', 0}}
/* rows: the argument that n is the first dimension of; table: the page table; pool: the pool of keys, the other follows it */
static const struct { const char* name; int n_args, rows, table, pool; param p[MAX_ARGS]; } operators[N_OPERATORS] = {
    /* transform, q, k, tok_pos, q_out, k_out */
    [QK_NORM_ROPE] = {"novakv_qk_norm_rope", 6, 3, -1, -1,
        {{'h', 0}, {'Q', 1}, {'s', 1}, {'K', 2}, {'s', 2}, {'i', 3}, {'N', 0}, {'Q', 4}, {'s', 4}, {'K', 5}, {'s', 5}, {'S', 0}}},
    /* transform, k_new, v_new, tok_seq, tok_pos, k_pages, v_pages, page_table, seq_lens, q, q_out */
    [BF16_APPEND] = {"novakv_bf16_append", 11, 1, 7, 5, APPEND_PARAMS('b')},
    [INT4_APPEND] = {"novakv_int4_append", 11, 1, 7, 5, APPEND_PARAMS('c')},
    /* tok_seq, tok_pos, k_pages, v_pages, page_table, k_out, v_out */
    [INT4_GATHER] = {"novakv_int4_gather", 7, 0, 4, 2,
        {{'i', 0}, {'i', 1}, {'N', 0}, {'c', 2}, {'c', 3}, {'0', 2}, {'t', 4}, {'1', 4}, {'0', 4}, {'e', 5}, {'e', 6}, {'T', 5}, {'S', 0}}},
    /* q, k_pages, v_pages, page_table, seq_lens, out, workspace, sm_scale, window, sink_logits */
    [INT4_DECODE] = {"novakv_int4_decode_attention", 10, 0, 3, 1,
        {{'q', 0}, {'c', 1}, {'c', 2}, {'0', 1}, {'t', 3}, {'1', 3}, {'l', 4}, {'N', 0}, {'F', 7}, {'I', 8}, {'f', 9}, {'o', 5}, {'T', 5}, {'w', 6}, {'B', 6}, {'S', 0}}},
};
static PyObject *bfloat16, *int32, *uint8;                 /* of torch, given by bind_operators() */

typedef struct {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    int entry;
    void* fn;
    long device, hq, hkv, d;
    PyObject* py_device;
} Operator;

static int refuse(int op, int arg, const char* what) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: argument %d %s", operators[op].name, arg + 1, what);
    return -1;
}
/* x.name() as an integer */
static long method_int(PyObject* x, PyObject* name) {
    PyObject* n = PyObject_CallMethodNoArgs(x, name);
    if (!n) return -1;
    const long v = n == Py_True ? 1 : n == Py_False ? 0 : PyLong_AsLong(n);
    Py_DECREF(n);
    return v;
}
/* sizes or strides of x into v (the first `most`); their number, or -1 */
static int dims_of(PyObject* s, long long* v, int most) {
    int n = -1;
    if (s && PyTuple_Check(s)) {
        n = (int)PyTuple_GET_SIZE(s);
        for (int i = 0; i < n && i < most; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
    }
    Py_XDECREF(s);
    return n;
}
/* What a call asks an argument for, once: an attribute of a tensor is a tenth of a microsecond. */
typedef struct { long long size[4], stride[3]; int dims; } sizes;
static int sizes_of(PyObject* x, sizes* z) {
    if (z->dims >= 0) return 0;
    z->dims = dims_of(PyObject_GetAttr(x, s_shape), z->size, 4);
    if (z->dims < 0 && !PyErr_Occurred()) PyErr_SetString(PyExc_AttributeError, "shape");
    return z->dims < 0 ? -1 : 0;
}
static int is_dtype(PyObject* x, PyObject* a, PyObject* b) {
    PyObject* t = PyObject_GetAttr(x, s_dtype);
    Py_XDECREF(t);
    return t && (t == a || t == b);
}
/* what is asked of argument `arg`; n: rows of the call, table_rows, pool_pages of its page table and its first pool */
static int check(const Operator* e, char kind, int arg, PyObject* x, sizes* z, long long n, long long table_rows, long long pool_pages) {
    const int op = e->entry;
    if (method_int(x, s_get_device) != e->device || PyErr_Occurred()) return refuse(op, arg, "has to be a tensor on the context's device");
    if (kind != 'w' && sizes_of(x, z)) return -1;
    const long long* v = z->size;
    switch (kind) {
        case 'q': case 'Q': case 'k': case 'K': {
            const long heads = kind == 'q' || kind == 'Q' ? e->hq : e->hkv;
            if (!is_dtype(x, bfloat16, bfloat16)) return refuse(op, arg, "has to be bfloat16");
            if (z->dims != 3 || v[0] != n || v[1] != heads || v[2] != e->d) return refuse(op, arg, "has to be rows [n][heads][head_dim]");
            if (dims_of(PyObject_CallMethodNoArgs(x, s_stride), z->stride, 3) != 3 || z->stride[2] != 1 || (z->stride[1] != e->d && heads > 1))
                return refuse(op, arg, "has to have contiguous heads");
            /* (decode attention takes no stride) */
            if (kind == 'q' && n > 1 && z->stride[0] != heads * e->d) return refuse(op, arg, "has to be contiguous");
            return 0;
        }
        case 'e': case 'o':
            if (!is_dtype(x, bfloat16, float32)) return refuse(op, arg, "has to be bfloat16 or float32");
            if (z->dims != 3 || v[0] != n || v[1] != (kind == 'o' ? e->hq : e->hkv) || v[2] != e->d) return refuse(op, arg, "has to be rows [n][heads][head_dim]");
            break;
        case 'i':
            if (!is_dtype(x, int32, int32) || z->dims != 1 || v[0] != n) return refuse(op, arg, "has to be int32, one for each row");
            break;
        case 't':
            if (!is_dtype(x, int32, int32) || z->dims != 2) return refuse(op, arg, "has to be an int32 table [sequences][pages]");
            break;
        case 'l':
            if (!is_dtype(x, int32, int32) || z->dims != 1 || v[0] != table_rows) return refuse(op, arg, "has to be int32, one for each row of the page table");
            break;
        case 'f':
            if (!is_dtype(x, float32, float32) || z->dims != 1 || v[0] != e->hq) return refuse(op, arg, "has to be float32, one for each query head");
            break;
        case 'b': case 'c': {                              /* [pages] and any dimensions behind, of a page's bytes in all */
            long long page = kind == 'b' ? 2 : 1;
            for (int i = 1; i < z->dims && i < 4; ++i) page *= v[i];
            const long long row = kind == 'b' ? e->d * 2 : e->d / 2 + e->d / 64 * 4;
            if (!is_dtype(x, kind == 'b' ? bfloat16 : uint8, NULL) || z->dims < 2 || z->dims > 4 || v[0] != pool_pages || page != e->hkv * 64 * row)
                return refuse(op, arg, "has to be a pool of this cache's pages, as many as the keys' pool");
            break;
        }
        default: break;
    }
    if (method_int(x, s_is_contiguous) != 1) return refuse(op, arg, "has to be contiguous");
    return 0;
}

static novakv_status call_operator(int entry, void* fn, novakv_ctx* c, const long long* a, float f) {
#define I(i) ((int)a[i])
#define V(i) ((void*)(uintptr_t)a[i])
    switch (entry) {
        case QK_NORM_ROPE:
            return ((__typeof__(&novakv_qk_norm_rope))fn)(c, V(0), V(1), a[2], V(3), a[4], V(5), I(6), V(7), a[8], V(9), a[10], V(11));
        case BF16_APPEND:
        case INT4_APPEND:
            return ((__typeof__(&novakv_int4_append))fn)(c, V(0), V(1), a[2], V(3), a[4], V(5), V(6), I(7), V(8), V(9), I(10), V(11), I(12), I(13), V(14), V(15), a[16],
                                                         V(17), a[18], V(19));
        case INT4_GATHER:
            return ((__typeof__(&novakv_int4_gather))fn)(c, V(0), V(1), I(2), V(3), V(4), I(5), V(6), I(7), I(8), V(9), V(10), I(11), V(12));
        default:
            return ((__typeof__(&novakv_int4_decode_attention))fn)(c, V(0), V(1), V(2), I(3), V(4), I(5), V(6), I(7), f, I(9), V(10), V(11), I(12), V(13), (size_t)a[14], V(15));
    }
#undef I
#undef V
}

/* operator(handle, arguments...) -> status */
static PyObject* operator_call(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* kwnames) {
    const Operator* e = (const Operator*)self;
    const int op = e->entry;
    if (kwnames || PyVectorcall_NARGS(nargsf) != operators[op].n_args + 1) {
        PyErr_Format(PyExc_TypeError, "%s: a context and %d positional arguments", operators[op].name, operators[op].n_args);
        return NULL;
    }
    const unsigned long long ctx = args[0] == Py_None ? 0 : PyLong_AsUnsignedLongLong(args[0]);
    if (PyErr_Occurred()) return NULL;
    sizes z[MAX_ARGS];
    for (int i = 0; i < operators[op].n_args; ++i) z[i].dims = -1;
    const int asked[3] = {operators[op].rows, operators[op].table, operators[op].pool};
    long long first[3] = {0, 0, 0};                        /* shape[0] of each */
    for (int i = 0; i < 3; ++i) {
        if (asked[i] < 0) continue;
        if (sizes_of(args[1 + asked[i]], &z[asked[i]])) return NULL;
        if (z[asked[i]].dims < 1) { refuse(op, asked[i], "has no dimension"); return NULL; }
        first[i] = z[asked[i]].size[0];
    }
    const long long n = first[0], table_rows = first[1], pool_pages = first[2];
    if (op == INT4_DECODE && n != table_rows) { refuse(op, operators[op].table, "has to have one row for each query"); return NULL; }
    if (n > INT_MAX || pool_pages > INT_MAX) { refuse(op, 0, "is too large"); return NULL; }
    long long a[MAX_ARGS];
    float f = 0.f;
    const param* p = operators[op].p;
    for (int i = 0; i < MAX_ARGS && p[i].kind; ++i) {
        const int arg = p[i].arg;
        PyObject* x = args[1 + arg];
        unsigned long long u = 0;
        a[i] = 0;
        switch (p[i].kind) {
            case 'Q': case 'K': case 'f':
                if (x == Py_None) break;                   /* fall through */
            case 'q': case 'k': case 'e': case 'o': case 'i': case 't': case 'l': case 'b': case 'c': case 'w':
                if (x == Py_None) { refuse(op, arg, "is missing"); return NULL; }
                if (check(e, p[i].kind, arg, x, &z[arg], n, table_rows, pool_pages) || pointer_of(x, &u)) return NULL;
                a[i] = (long long)u;
                break;
            case 'h': case 'H':
                if (x == Py_None && p[i].kind == 'h') { refuse(op, arg, "is missing"); return NULL; }
                if (pointer_of(x, &u)) return NULL;
                a[i] = (long long)u;
                break;
            case 's':
                if (x == Py_None) break;                   /* (behind its rows: they have been looked at) */
                a[i] = n > 1 ? z[arg].stride[0] : e->hq * e->d;        /* (of a single row any stride is one) */
                break;
            case 'N': a[i] = n; break;
            case '0': case '1':                            /* (what the C call takes as an int) */
                a[i] = z[arg].size[p[i].kind - '0'];
                if (a[i] > INT_MAX) { refuse(op, arg, "is too large"); return NULL; }
                break;
            case 'I':
                if (as_int(x, 0, &a[i])) return NULL;
                if (a[i] > INT_MAX || a[i] < INT_MIN) { refuse(op, arg, "is out of range"); return NULL; }
                break;
            case 'F': f = (float)PyFloat_AsDouble(x); break;
            case 'T': a[i] = is_dtype(x, float32, float32); break;
            case 'B': { PyObject* b = PyObject_GetAttr(x, s_nbytes); if (!b) return NULL; a[i] = PyLong_AsLongLong(b); Py_DECREF(b); break; }
            default: {
                PyObject* s = PyObject_CallOneArg(get_stream, e->py_device);
                if (!s) return NULL;
                a[i] = (long long)PyLong_AsUnsignedLongLong(s);
                Py_DECREF(s);
            }
        }
        if (PyErr_Occurred()) return NULL;
    }
    if (op == INT4_GATHER) {                               /* both outputs of one type */
        if (is_dtype(args[6], float32, float32) != is_dtype(args[7], float32, float32)) { refuse(op, 6, "has to have the type of the keys' output"); return NULL; }
    }
    novakv_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call_operator(op, e->fn, (novakv_ctx*)(uintptr_t)ctx, a, f);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

static void operator_dealloc(PyObject* self) {
    Py_XDECREF(((Operator*)self)->py_device);
    PyObject_Free(self);
}

static PyTypeObject OperatorType = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "_novakv_calls.Operator",
    .tp_basicsize = sizeof(Operator),
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL,
    .tp_vectorcall_offset = offsetof(Operator, vectorcall),
    .tp_call = PyVectorcall_Call,
    .tp_dealloc = operator_dealloc,
};

/* bind_operators(handle of the opened library, device, Hq, Hkv, head_dim, (torch.bfloat16, torch.int32, torch.uint8)) -> {name: operator} */
static PyObject* bind_operators(PyObject* self, PyObject* args) {
    PyObject *handle, *a, *b, *c;
    long device, hq, hkv, d;
    if (!PyArg_ParseTuple(args, "Ollll(OOO)", &handle, &device, &hq, &hkv, &d, &a, &b, &c)) return NULL;
    void* h = PyLong_AsVoidPtr(handle);
    if (PyErr_Occurred()) return NULL;
    if (!get_stream) { PyErr_SetString(PyExc_RuntimeError, "setup() comes first"); return NULL; }
    Py_INCREF(a); Py_INCREF(b); Py_INCREF(c);
    Py_XSETREF(bfloat16, a);
    Py_XSETREF(int32, b);
    Py_XSETREF(uint8, c);
    PyObject* dict = PyDict_New();
    for (int i = 0; dict && i < N_OPERATORS; ++i) {
        void* fn = dlsym(h, operators[i].name);
        Operator* e = fn ? PyObject_New(Operator, &OperatorType) : NULL;
        if (!fn) PyErr_Format(PyExc_RuntimeError, "the library lacks %s", operators[i].name);
        if (e) {
            e->vectorcall = operator_call; e->entry = i; e->fn = fn;
            e->device = device; e->hq = hq; e->hkv = hkv; e->d = d;
            e->py_device = PyLong_FromLong(device);
        }
        if (!e || !e->py_device || PyDict_SetItemString(dict, operators[i].name, (PyObject*)e)) Py_CLEAR(dict);
        Py_XDECREF((PyObject*)e);
    }
    return dict;
}

/* setup(current stream of a device, current device, torch.float32): what the calls ask torch for */
static PyObject* setup(PyObject* self, PyObject* args) {
    PyObject *a, *b, *c;
    if (!PyArg_ParseTuple(args, "OOO", &a, &b, &c)) return NULL;
    Py_INCREF(a); Py_INCREF(b); Py_INCREF(c);
    Py_XSETREF(get_stream, a);
    Py_XSETREF(get_device, b);
    Py_XSETREF(float32, c);
    Py_RETURN_NONE;
}
/* bind(handle of the opened library) -> {name: entry} */
static PyObject* bind(PyObject* self, PyObject* handle) {
    void* h = PyLong_AsVoidPtr(handle);
    if (PyErr_Occurred()) return NULL;
    if (!get_stream) { PyErr_SetString(PyExc_RuntimeError, "setup() comes first"); return NULL; }
    PyObject* d = PyDict_New();
    for (int i = 0; d && i < N_ENTRIES; ++i) {
        void* fn = dlsym(h, entries[i].name);
        Entry* e = fn ? PyObject_New(Entry, &EntryType) : NULL;
        if (!fn) PyErr_Format(PyExc_RuntimeError, "the library lacks %s", entries[i].name);
        if (e) { e->vectorcall = entry_call; e->entry = i; e->fn = fn; }
        if (!e || PyDict_SetItemString(d, entries[i].name, (PyObject*)e)) Py_CLEAR(d);
        Py_XDECREF((PyObject*)e);
    }
    return d;
}

static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, NULL}, {"bind", bind, METH_O, NULL},
                                {"bind_operators", bind_operators, METH_VARARGS, NULL}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_novakv_calls", NULL, -1, methods};

PyMODINIT_FUNC PyInit__novakv_calls(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_stride = PyUnicode_InternFromString("stride");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    if (!s_data_ptr || !s_shape || !s_dtype || !s_nbytes || !s_stride || !s_get_device || !s_is_contiguous || PyType_Ready(&EntryType) < 0 ||
        PyType_Ready(&OperatorType) < 0) return NULL;
    return PyModule_Create(&module);
}
