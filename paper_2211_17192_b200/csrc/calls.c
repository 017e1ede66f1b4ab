/* The checks and the calls of the entry points that a host makes once per decision (sampling) or several times per decoder block
 * (the 8-bit operators), from Python.
 *
 * A lone decision keeps the GPU busy for 8 us; checking seven tensors in Python and a call through ctypes took the host 10.5.  Here
 * the same questions are asked of the same objects (is_cuda, dtype, is_contiguous(), shape, data_ptr()) from C, and the library
 * is called through its address: 4 x 8192 logits, call after call, 10.5 -> 9.6 us, 7.7 where the GPU
 * need not wait between two of them.
 * Whatever is not the plain case - another type, a missing tensor, a shape that does not fit - is answered with None and
 * nothing done: binding.py then makes the call itself and says what is wrong. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*verify_fn)(const float*, const float*, const int32_t*, const float*, int, int, int, float, float, int, float, int32_t*,
                         int32_t*, void*, size_t, void*);
typedef int (*sample_fn)(const float*, const float*, int, int, float, int32_t*, void*);

static verify_fn g_verify;
static sample_fn g_sample;
static PyObject *g_float32, *g_int32, *g_uint8;
static PyObject *s_is_cuda, *s_dtype, *s_is_contiguous, *s_shape, *s_data_ptr, *s_numel;

/* The address of a contiguous CUDA tensor of this type; its sizes in dims[n] (n < 0: not asked for).  0: something else. */
static int tensor(PyObject* t, PyObject* dtype, int n, Py_ssize_t* dims, void** address) {
    PyObject* v = PyObject_GetAttr(t, s_is_cuda);
    if (!v) return 0;
    Py_DECREF(v);
    if (v != Py_True) return 0;
    if (!(v = PyObject_GetAttr(t, s_dtype))) return 0;
    Py_DECREF(v);
    if (v != dtype) return 0;
    if (!(v = PyObject_CallMethodNoArgs(t, s_is_contiguous))) return 0;
    Py_DECREF(v);
    if (v != Py_True) return 0;
    if (n >= 0) {
        int fits;
        if (!(v = PyObject_GetAttr(t, s_shape))) return 0;
        fits = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == n;
        for (int i = 0; fits && i < n; ++i) {
            dims[i] = PyLong_AsSsize_t(PyTuple_GET_ITEM(v, i));
            if (dims[i] < 0 || dims[i] > INT32_MAX) fits = 0;
        }
        Py_DECREF(v);
        if (!fits) return 0;
    }
    if (!(v = PyObject_CallMethodNoArgs(t, s_data_ptr))) return 0;
    *address = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

static int number(PyObject* o, double* out) {
    if (!PyFloat_Check(o) && !PyLong_Check(o)) return 0;
    *out = PyFloat_AsDouble(o);
    return !PyErr_Occurred();
}

static PyObject* not_plain(void) {
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* verify(target, draft, tokens, uniforms, n_accepted, next_token, workspace, temperature, lenience, top_k, top_p, stream) -> status */
static PyObject* verify(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    void *target, *draft, *tokens, *uniforms, *accepted, *next, *workspace, *stream;
    Py_ssize_t t[3], q[3], x[2], u[2];
    double temperature, lenience, top_p;
    long top_k;
    size_t bytes;
    PyObject* v;
    int status;
    (void)self;
    if (count != 12 || !g_verify) return not_plain();
    if (!tensor(a[0], g_float32, 3, t, &target) || !tensor(a[1], g_float32, 3, q, &draft) || !tensor(a[2], g_int32, 2, x, &tokens) ||
        !tensor(a[3], g_float32, 2, u, &uniforms) || !tensor(a[4], g_int32, -1, NULL, &accepted) ||
        !tensor(a[5], g_int32, -1, NULL, &next) || !tensor(a[6], g_uint8, -1, NULL, &workspace))
        return not_plain();
    if (t[1] < 2 || q[0] != t[0] || q[1] != t[1] - 1 || q[2] != t[2] || x[0] != t[0] || x[1] != t[1] - 1 || u[0] != t[0] || u[1] != t[1])
        return not_plain();
    if (!number(a[7], &temperature) || !number(a[8], &lenience) || !PyLong_Check(a[9]) || !number(a[10], &top_p)) return not_plain();
    top_k = PyLong_AsLong(a[9]);
    if (PyErr_Occurred() || top_k < INT32_MIN || top_k > INT32_MAX) return not_plain();
    if (!(v = PyObject_CallMethodNoArgs(a[6], s_numel))) return not_plain();
    bytes = PyLong_AsSize_t(v);
    Py_DECREF(v);
    stream = PyLong_AsVoidPtr(a[11]);
    if (PyErr_Occurred()) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_verify((const float*)target, (const float*)draft, (const int32_t*)tokens, (const float*)uniforms, (int)t[0], (int)t[1] - 1,
                      (int)t[2], (float)temperature, (float)lenience, (int)top_k, (float)top_p, (int32_t*)accepted, (int32_t*)next,
                      workspace, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* sample(logits, uniforms, temperature, tokens, stream) -> status */
static PyObject* sample(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    void *logits, *uniforms, *tokens, *stream;
    Py_ssize_t l[2];
    double temperature;
    int status;
    (void)self;
    if (count != 5 || !g_sample) return not_plain();
    if (!tensor(a[0], g_float32, 2, l, &logits) || !tensor(a[1], g_float32, -1, NULL, &uniforms) || !number(a[2], &temperature) ||
        !tensor(a[3], g_int32, -1, NULL, &tokens))
        return not_plain();
    stream = PyLong_AsVoidPtr(a[4]);
    if (PyErr_Occurred()) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_sample((const float*)logits, (const float*)uniforms, (int)l[0], (int)l[1], (float)temperature, (int32_t*)tokens, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* ---- the 8-bit operators ----
 * A call with all its outputs given, as a serving loop makes it: norm of one row of 768 22.7 -> 5.7 us call after call, append and read
 * of 32 x 7 rows 71.7 -> 12.2, attention with its workspace 31.4 -> 8.9 (the checks in Python are a microsecond or two per tensor). */
typedef int (*quantize_fn)(const void*, int, int, int, void*, float*, void*);
typedef int (*norm_fn)(const void*, int, const void*, void*, int, const float*, float, int, int, void*, float*, void*);
typedef int (*linear_fn)(const void*, const float*, const void*, const float*, const float*, int, const void*, void*, int, int, int, int, void*);
typedef int (*append_fn)(const void*, const void*, const void*, int, int64_t, int64_t, int64_t, int, int, int, int, int, const int32_t*, const int32_t*,
                         const float*, int, void*, void*, float*, int, int, int, const int32_t*, int, void*);
typedef int (*read_fn)(const void*, const float*, int, int, int, int, int, const int32_t*, int, int, int, const int32_t*, const int32_t*, void*, void*, int, void*);
typedef int (*attention_fn)(const void*, int, int64_t, const void*, const float*, int, int, int, const int32_t*, int, const int32_t*, int, int, int, int, int,
                            float, void*, void*, size_t, void*);
enum { FP32, BF16, FP16, E4M3, INT8, INT32, UINT8, KINDS };  /* (the first five as the library numbers them) */
#define ONE(kind) (1u << (kind))
#define FLOATS (ONE(FP32) | ONE(BF16) | ONE(FP16))

static struct {
    quantize_fn quantize;
    norm_fn norm;
    linear_fn linear;
    append_fn append;
    read_fn read;
    attention_fn attention;
} g_ops;
static PyObject* g_kinds[KINDS];
static PyObject *s_get_device, *s_stride;

typedef struct {
    void* at;
    int kind, n;
    Py_ssize_t dims[5];
} operand;

/* The address, type (one of the set) and n sizes of a tensor of the current GPU; with `row` it may be [B, rows, heads, d] with dense
 * heads and one distance between rows, which goes there, and else it is contiguous.  0: something else. */
static int look(PyObject* t, unsigned kinds, int n, long device, operand* o, int64_t* row) {
    long where;
    int fits;
    PyObject* v = PyObject_CallMethodNoArgs(t, s_get_device);  /* (-1 for one that is on no GPU) */
    if (!v) return 0;
    where = PyLong_AsLong(v);
    Py_DECREF(v);
    if (where != device) return 0;
    if (!(v = PyObject_GetAttr(t, s_dtype))) return 0;
    Py_DECREF(v);
    for (o->kind = 0; o->kind < KINDS && v != g_kinds[o->kind];) ++o->kind;
    if (o->kind == KINDS || !(kinds & ONE(o->kind))) return 0;
    if (!(v = PyObject_GetAttr(t, s_shape))) return 0;
    fits = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == n;
    for (int i = 0; fits && i < n; ++i) {
        o->dims[i] = PyLong_AsSsize_t(PyTuple_GET_ITEM(v, i));
        if (o->dims[i] < 1 || o->dims[i] > INT32_MAX) fits = 0;
    }
    Py_DECREF(v);
    if (!fits) return 0;
    o->n = n;
    if (row) {
        Py_ssize_t s[4];
        if (!(v = PyObject_CallMethodNoArgs(t, s_stride))) return 0;
        fits = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 4;
        for (int i = 0; fits && i < 4; ++i) s[i] = PyLong_AsSsize_t(PyTuple_GET_ITEM(v, i));
        Py_DECREF(v);
        if (!fits || PyErr_Occurred() || s[3] != 1 || s[2] != o->dims[3]) return 0;
        *row = o->dims[1] > 1 ? s[1] : o->dims[0] > 1 ? s[0] : o->dims[2] * o->dims[3];  /* (a lone row's own stride may be anything) */
        if (o->dims[0] > 1 && o->dims[1] > 1 && s[0] != o->dims[1] * s[1]) return 0;
    } else {
        if (!(v = PyObject_CallMethodNoArgs(t, s_is_contiguous))) return 0;
        Py_DECREF(v);
        if (v != Py_True) return 0;
    }
    if (!(v = PyObject_CallMethodNoArgs(t, s_data_ptr))) return 0;
    o->at = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
/* The same for one that may be None (address NULL), with the sizes it has to have. */
static int look_as(PyObject* t, unsigned kinds, long device, operand* o, int optional, int n, Py_ssize_t d0, Py_ssize_t d1, Py_ssize_t d2, Py_ssize_t d3) {
    const Py_ssize_t want[4] = {d0, d1, d2, d3};
    if (optional && t == Py_None) {
        o->at = NULL;
        return 1;
    }
    if (!look(t, kinds, n, device, o, NULL)) return 0;
    for (int i = 0; i < n; ++i)
        if (o->dims[i] != want[i]) return 0;
    return 1;
}
static int whole(PyObject* o, long* out) {
    if (!PyLong_Check(o)) return 0;
    *out = PyLong_AsLong(o);
    return !PyErr_Occurred();
}
static int address(PyObject* o, void** out) {
    *out = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

/* quantize(x, codes, scales, device, stream) -> status */
static PyObject* quantize(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    operand x, codes, scales;
    long device;
    void* stream;
    int status;
    (void)self;
    if (count != 5 || !g_ops.quantize || !whole(a[3], &device) || !address(a[4], &stream)) return not_plain();
    if (!look(a[0], FLOATS, 2, device, &x, NULL) || !look_as(a[1], ONE(E4M3), device, &codes, 0, 2, x.dims[0], x.dims[1], 0, 0) ||
        !look_as(a[2], ONE(FP32), device, &scales, 0, 1, x.dims[0], 0, 0, 0))
        return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_ops.quantize(x.at, x.kind, (int)x.dims[0], (int)x.dims[1], codes.at, (float*)scales.at, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* norm(x, gain, eps, residual or None, h or None, codes, scales, device, stream) -> status */
static PyObject* norm(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    operand x, gain, residual, h, codes, scales;
    long device;
    double eps;
    void* stream;
    int status;
    (void)self;
    if (count != 9 || !g_ops.norm || !number(a[2], &eps) || !whole(a[7], &device) || !address(a[8], &stream)) return not_plain();
    if (!look(a[0], FLOATS, 2, device, &x, NULL) || !look_as(a[1], ONE(FP32), device, &gain, 0, 1, x.dims[1], 0, 0, 0) ||
        !look_as(a[3], ONE(FP32) | ONE(x.kind), device, &residual, 1, 2, x.dims[0], x.dims[1], 0, 0) ||
        !look_as(a[4], ONE(FP32) | ONE(x.kind), device, &h, 1, 2, x.dims[0], x.dims[1], 0, 0) ||
        !look_as(a[5], ONE(E4M3), device, &codes, 0, 2, x.dims[0], x.dims[1], 0, 0) || !look_as(a[6], ONE(FP32), device, &scales, 0, 1, x.dims[0], 0, 0, 0))
        return not_plain();
    if (a[3] != Py_None && (a[4] == Py_None || residual.kind != h.kind)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_ops.norm(x.at, x.kind, residual.at, h.at, a[4] != Py_None ? h.kind : FP32, (const float*)gain.at, (float)eps, (int)x.dims[0], (int)x.dims[1], codes.at,
                        (float*)scales.at, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* linear(x, x_scales, w, w_scales, bias or None, act, residual or None, y, device, stream) -> status */
static PyObject* linear(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    operand x, xs, w, ws, bias, residual, y;
    long device, act;
    void* stream;
    int status;
    (void)self;
    if (count != 10 || !g_ops.linear || !whole(a[5], &act) || !whole(a[8], &device) || !address(a[9], &stream)) return not_plain();
    if (!look(a[0], ONE(E4M3), 2, device, &x, NULL) || !look(a[2], ONE(E4M3), 2, device, &w, NULL) || !look(a[7], FLOATS, 2, device, &y, NULL) ||
        !look_as(a[1], ONE(FP32), device, &xs, 0, 1, x.dims[0], 0, 0, 0) || !look_as(a[3], ONE(FP32), device, &ws, 0, 1, w.dims[0], 0, 0, 0) ||
        !look_as(a[4], ONE(FP32), device, &bias, 1, 1, w.dims[0], 0, 0, 0) || !look_as(a[6], ONE(y.kind), device, &residual, 1, 2, y.dims[0], y.dims[1], 0, 0))
        return not_plain();
    if (x.dims[1] != w.dims[1] || y.dims[0] != x.dims[0] || y.dims[1] * (act >= 3 ? 2 : 1) != w.dims[0] || act < 0 || act > 4) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_ops.linear(x.at, (const float*)xs.at, w.at, (const float*)ws.at, (const float*)bias.at, (int)act, residual.at, y.at, y.kind, (int)x.dims[0],
                          (int)y.dims[1], (int)x.dims[1], stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* A pool, its scales (None beside a 16-bit one) and its page table. */
typedef struct {
    operand pool, scales, table;
} cache;
static int look_cache(PyObject* pool, PyObject* scales, PyObject* table, long device, cache* c) {
    if (!look(pool, ONE(FP16) | ONE(BF16) | ONE(E4M3) | ONE(INT8), 5, device, &c->pool, NULL) || c->pool.dims[1] != 2) return 0;
    if (c->pool.kind == E4M3 || c->pool.kind == INT8) {
        if (!look_as(scales, ONE(FP32), device, &c->scales, 0, 4, c->pool.dims[0], 2, c->pool.dims[2], c->pool.dims[3])) return 0;
    } else {
        if (scales != Py_None) return 0;
        c->scales.at = NULL;
    }
    return look(table, ONE(INT32), 2, device, &c->table, NULL);
}

/* append(k, v, pool, scales, page_table, start, counts, rope, q, q_out, device, stream) -> status */
static PyObject* append(PyObject* self, PyObject* const* arg, Py_ssize_t count) {
    operand k, v, start, counts, rope, q, q_out;
    cache c;
    long device;
    int64_t ks, vs, qs = 0;
    void* stream;
    int status;
    (void)self;
    if (count != 12 || !g_ops.append || !whole(arg[10], &device) || !address(arg[11], &stream)) return not_plain();
    if (!look(arg[0], FLOATS, 4, device, &k, &ks) || !look(arg[1], ONE(k.kind), 4, device, &v, &vs) || !look_cache(arg[2], arg[3], arg[4], device, &c) ||
        !look_as(arg[5], ONE(INT32), device, &start, 0, 1, k.dims[0], 0, 0, 0) || !look_as(arg[6], ONE(INT32), device, &counts, 1, 1, k.dims[0], 0, 0, 0))
        return not_plain();
    for (int i = 0; i < 4; ++i)
        if (v.dims[i] != k.dims[i]) return not_plain();
    if (c.pool.dims[2] != k.dims[2] || c.pool.dims[4] != k.dims[3] || c.table.dims[0] != k.dims[0]) return not_plain();
    rope.at = q.at = q_out.at = NULL;
    rope.dims[0] = q.dims[2] = 0;
    if (arg[7] != Py_None && (!look(arg[7], ONE(FP32), 3, device, &rope, NULL) || 2 * rope.dims[1] != k.dims[3] || rope.dims[2] != 2)) return not_plain();
    if (arg[8] != Py_None) {
        if (!look(arg[8], ONE(k.kind), 4, device, &q, &qs) || q.dims[0] != k.dims[0] || q.dims[1] != k.dims[1] || q.dims[3] != k.dims[3]) return not_plain();
        if (!look_as(arg[9], ONE(k.kind), device, &q_out, 0, 4, q.dims[0], q.dims[1], q.dims[2], q.dims[3])) return not_plain();
    } else if (arg[9] != Py_None) {
        return not_plain();
    }
    Py_BEGIN_ALLOW_THREADS
    status = g_ops.append(q.at, k.at, v.at, k.kind, qs, ks, vs, (int)q.dims[2], (int)k.dims[2], (int)k.dims[3], (int)k.dims[0], (int)k.dims[1],
                          (const int32_t*)start.at, (const int32_t*)counts.at, (const float*)rope.at, (int)rope.dims[0], q_out.at, c.pool.at, (float*)c.scales.at,
                          c.pool.kind, (int)c.pool.dims[0], (int)c.pool.dims[3], (const int32_t*)c.table.at, (int)c.table.dims[1], stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* read(pool, scales, page_table, start, rows, counts, k, v, device, stream) -> status */
static PyObject* read_rows(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    operand start, counts, k, v;
    cache c;
    long device, rows;
    void* stream;
    int status;
    (void)self;
    if (count != 10 || !g_ops.read || !whole(a[4], &rows) || !whole(a[8], &device) || !address(a[9], &stream)) return not_plain();
    if (!look_cache(a[0], a[1], a[2], device, &c) || !look_as(a[3], ONE(INT32), device, &start, 0, 1, c.table.dims[0], 0, 0, 0) ||
        !look_as(a[5], ONE(INT32), device, &counts, 1, 1, c.table.dims[0], 0, 0, 0) ||
        !look_as(a[6], FLOATS, device, &k, 0, 4, c.table.dims[0], rows, c.pool.dims[2], c.pool.dims[4]) ||
        !look_as(a[7], ONE(k.kind), device, &v, 0, 4, c.table.dims[0], rows, c.pool.dims[2], c.pool.dims[4]))
        return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_ops.read(c.pool.at, (const float*)c.scales.at, c.pool.kind, (int)c.pool.dims[0], (int)c.pool.dims[3], (int)c.pool.dims[2], (int)c.pool.dims[4],
                        (const int32_t*)c.table.at, (int)c.table.dims[1], (int)c.table.dims[0], (int)rows, (const int32_t*)start.at, (const int32_t*)counts.at,
                        k.at, v.at, k.kind, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* attention(q, pool, scales, page_table, lengths, scale, out, workspace, device, stream) -> status */
static PyObject* attention(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    operand q, lengths, out, workspace;
    cache c;
    long device;
    int64_t qs;
    double scale;
    void* stream;
    int status;
    (void)self;
    if (count != 10 || !g_ops.attention || !number(a[5], &scale) || !whole(a[8], &device) || !address(a[9], &stream)) return not_plain();
    if (!look(a[0], ONE(BF16) | ONE(FP16), 4, device, &q, &qs) || !look_cache(a[1], a[2], a[3], device, &c) ||
        !look_as(a[4], ONE(INT32), device, &lengths, 0, 1, q.dims[0], 0, 0, 0) ||
        !look_as(a[6], ONE(q.kind), device, &out, 0, 4, q.dims[0], q.dims[1], q.dims[2], q.dims[3]) || !look(a[7], ONE(UINT8), 1, device, &workspace, NULL))
        return not_plain();
    if (c.table.dims[0] != q.dims[0] || c.pool.dims[4] != q.dims[3] || q.dims[2] % c.pool.dims[2]) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    status = g_ops.attention(q.at, q.kind, qs, c.pool.at, (const float*)c.scales.at, c.pool.kind, (int)c.pool.dims[0], (int)c.pool.dims[3],
                             (const int32_t*)c.table.at, (int)c.table.dims[1], (const int32_t*)lengths.at, (int)q.dims[0], (int)q.dims[1], (int)q.dims[2],
                             (int)c.pool.dims[2], (int)q.dims[3], (float)scale, out.at, workspace.at, (size_t)workspace.dims[0], stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* bind_operators((addresses of spec_quantize_fp8, spec_norm_fp8, spec_linear_fp8, spec_kv_append, spec_kv_read, spec_paged_attention),
 * (torch.float32, bfloat16, float16, float8_e4m3fn, int8, int32, uint8)) */
static PyObject* bind_operators(PyObject* self, PyObject* args) {
    PyObject *at[6], *kinds;
    (void)self;
    if (!PyArg_ParseTuple(args, "(OOOOOO)O!", &at[0], &at[1], &at[2], &at[3], &at[4], &at[5], &PyTuple_Type, &kinds)) return NULL;
    if (PyTuple_GET_SIZE(kinds) != KINDS) {
        PyErr_SetString(PyExc_ValueError, "seven types");
        return NULL;
    }
    g_ops.quantize = (quantize_fn)(uintptr_t)PyLong_AsVoidPtr(at[0]);
    g_ops.norm = (norm_fn)(uintptr_t)PyLong_AsVoidPtr(at[1]);
    g_ops.linear = (linear_fn)(uintptr_t)PyLong_AsVoidPtr(at[2]);
    g_ops.append = (append_fn)(uintptr_t)PyLong_AsVoidPtr(at[3]);
    g_ops.read = (read_fn)(uintptr_t)PyLong_AsVoidPtr(at[4]);
    g_ops.attention = (attention_fn)(uintptr_t)PyLong_AsVoidPtr(at[5]);
    if (PyErr_Occurred()) return NULL;
    for (int i = 0; i < KINDS; ++i) {
        g_kinds[i] = PyTuple_GET_ITEM(kinds, i);
        Py_INCREF(g_kinds[i]);
    }
    Py_RETURN_NONE;
}

/* bind(address of spec_verify_sample_truncated, of spec_sample, torch.float32, torch.int32, torch.uint8) */
static PyObject* bind(PyObject* self, PyObject* args) {
    PyObject *verify_at, *sample_at, *f, *i, *u;
    (void)self;
    if (!PyArg_ParseTuple(args, "OOOOO", &verify_at, &sample_at, &f, &i, &u)) return NULL;
    g_verify = (verify_fn)(uintptr_t)PyLong_AsVoidPtr(verify_at);
    g_sample = (sample_fn)(uintptr_t)PyLong_AsVoidPtr(sample_at);
    if (PyErr_Occurred()) return NULL;
    Py_INCREF(f);
    Py_INCREF(i);
    Py_INCREF(u);
    g_float32 = f;
    g_int32 = i;
    g_uint8 = u;
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, NULL},
    {"verify", (PyCFunction)(void (*)(void))verify, METH_FASTCALL, NULL},
    {"sample", (PyCFunction)(void (*)(void))sample, METH_FASTCALL, NULL},
    {"bind_operators", bind_operators, METH_VARARGS, NULL},
    {"quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, NULL},
    {"norm", (PyCFunction)(void (*)(void))norm, METH_FASTCALL, NULL},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, NULL},
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, NULL},
    {"read", (PyCFunction)(void (*)(void))read_rows, METH_FASTCALL, NULL},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_shape = PyUnicode_InternFromString("shape");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_stride = PyUnicode_InternFromString("stride");
    if (!s_is_cuda || !s_dtype || !s_is_contiguous || !s_shape || !s_data_ptr || !s_numel || !s_get_device || !s_stride) return NULL;
    return PyModule_Create(&module);
}
