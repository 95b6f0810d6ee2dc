/* Python front-end of the entry points that take no context (moe_gate, moe_add_rmsnorm, moe_project, moe_block_norm, moe_quantize_i8,
 * moe_project_i8, moe_balance_loss and the gradients).
 *
 * Their kernels run in a few microseconds, about what ctypes and Python need to look at ten tensors, so the checks and the
 * marshalling are done here with the CPython API: a tensor's dtype, device, shape, stride and address are read
 * through its public attributes (nothing of torch is linked), the entry points are called by the addresses that
 * binding.py hands over.  A check that fails raises ValueError; the status of the call is returned, or kOtherDevice if the
 * tensors' device is not the current one (the caller switches and calls again). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "faasmoe.h"

enum { kOtherDevice = 1 };

typedef int (*gate_fn)(const void*, int, int64_t, int, int, int, const moe_gating*, const float*, const int32_t*, const int32_t*, int,
                       int, int32_t*, float*, uint8_t*, int32_t*, void*);
typedef int (*norm_fn)(const void*, int64_t, const void*, int64_t, const void*, float, int, int, void*, int64_t, void*, int64_t, void*,
                       int64_t, float*, int, void*);
typedef int (*project_fn)(const void*, int64_t, const void*, int64_t, int, int, int, const void*, const void*, const float*, int, int,
                          const int32_t*, const int32_t*, int, const void*, int64_t, void*, int64_t, int, void*, int64_t, int32_t*, void*);
typedef int64_t (*workspace_fn)(int, int, int, int, int);
typedef int (*block_fn)(const void*, int64_t, const void*, int64_t, const void*, const void*, const void*, int64_t, const moe_block_rule*, int, int,
                        void*, int64_t, void*, int64_t, int8_t*, int64_t, float*, void*);
typedef int (*block_grad_fn)(const void*, int64_t, const void*, int64_t, const void*, const void*, const void*, int64_t, const moe_block_rule*, int,
                             int, const void*, int64_t, const void*, int64_t, void*, int64_t, void*, int64_t, void*, int64_t, float*, float*, void*,
                             int64_t, void*);
typedef int64_t (*block_workspace_fn)(int, int);
typedef int (*quantize_fn)(const void*, int64_t, int, int, int8_t*, int64_t, float*, void*);
typedef int (*project_i8_fn)(const int8_t*, int64_t, const float*, const int8_t*, int64_t, const float*, int, int, int, const float*, const void*,
                             int64_t, void*, int64_t, int, int32_t*, void*);
typedef int (*balance_fn)(const void*, int, int64_t, int, int, int, int, const int32_t*, const uint8_t*, const int32_t*, const int32_t*, int, int,
                          int32_t*, int32_t*, float*, float*, float*, void*, int64_t, int32_t*, void*);
typedef int64_t (*balance_workspace_fn)(int, int, int);
typedef int (*gate_grad_fn)(const void*, int, int64_t, int, int, int, const moe_gating*, const int32_t*, const float*, const uint8_t*, const int32_t*,
                            const int32_t*, int, int, const int32_t*, const int32_t*, const float*, const float*, void*, int64_t, int32_t*, void*);

static gate_fn f_gate;
static norm_fn f_norm;
static project_fn f_project;
static workspace_fn f_workspace;
static block_fn f_block;
static block_grad_fn f_block_grad;
static block_workspace_fn f_block_workspace;
static quantize_fn f_quantize;
static project_i8_fn f_project_i8;
static balance_fn f_balance;
static balance_workspace_fn f_balance_workspace;
static gate_grad_fn f_gate_grad;
static PyObject *t_f32, *t_bf16, *t_i32, *t_u8, *t_e4m3, *t_i8;          /* torch dtypes */
static PyObject *c_raw_stream, *c_get_device, *c_empty, *rule_type;      /* callables; the gating struct's class */
static PyObject *n_dtype, *n_device, *n_shape, *n_stride, *n_data_ptr, *n_is_contiguous, *n_type, *n_index, *n_cuda_stream;

/* what a call works on: the device of its first tensor, as an object and as an index */
typedef struct {
    const char* fn;
    PyObject* device;
    long index;
} Call;

static int fail(const Call* c, const char* name, const char* what, PyObject* t)
{
    PyObject* shape = t ? PyObject_GetAttr(t, n_shape) : NULL;
    PyObject* dtype = shape ? PyObject_GetAttr(t, n_dtype) : NULL;
    PyObject* device = dtype ? PyObject_GetAttr(t, n_device) : NULL;
    PyErr_Clear();
    if (device) {
        PyObject* dims = PySequence_List(shape);
        PyErr_Clear();
        PyErr_Format(PyExc_ValueError, "%s: %s %s, not %S of %S on %S", c->fn, name, what, dims ? dims : shape, dtype, device);
        Py_XDECREF(dims);
    } else {
        PyErr_Format(PyExc_ValueError, "%s: %s %s", c->fn, name, what);
    }
    Py_XDECREF(shape); Py_XDECREF(dtype); Py_XDECREF(device);
    return -1;
}

/* sizes of a tensor's dimensions; -1 with an exception, or the number of dimensions (at most 4 are written) */
static int sizes_of(PyObject* t, int64_t* sizes)
{
    PyObject* shape = PyObject_GetAttr(t, n_shape);
    if (!shape) return -1;
    if (!PyTuple_Check(shape)) { Py_DECREF(shape); PyErr_SetString(PyExc_TypeError, "a tensor is needed"); return -1; }
    const Py_ssize_t n = PyTuple_GET_SIZE(shape);
    for (Py_ssize_t i = 0; i < n && i < 4; ++i) sizes[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
    Py_DECREF(shape);
    return PyErr_Occurred() ? -1 : (int)n;
}

static int has(PyObject* t, PyObject* name, PyObject* want)        /* 1: the attribute is this object, 0: not, -1: exception */
{
    PyObject* v = PyObject_GetAttr(t, name);
    if (!v) return -1;
    const int r = v == want;
    Py_DECREF(v);
    return r;
}

static int on_device(const Call* c, PyObject* t)
{
    PyObject* d = PyObject_GetAttr(t, n_device);
    if (!d) return -1;
    const int r = d == c->device ? 1 : PyObject_RichCompareBool(d, c->device, Py_EQ);
    Py_DECREF(d);
    return r;
}

static int address_of(PyObject* t, void** p)
{
    PyObject* a = PyObject_CallMethodNoArgs(t, n_data_ptr);
    if (!a) return -1;
    *p = (void*)(uintptr_t)PyLong_AsUnsignedLongLong(a);
    Py_DECREF(a);
    return PyErr_Occurred() ? -1 : 0;
}

/* [rows, cols] matrix of `dtype` whose rows may be strided (None: a NULL pointer) */
static int matrix(const Call* c, PyObject* t, const char* name, int64_t rows, int64_t cols, PyObject* dtype, void** p, int64_t* ld)
{
    *p = NULL; *ld = 0;
    if (t == Py_None) return 0;
    int64_t size[4], step[2];
    const int n = sizes_of(t, size);
    if (n < 0) return -1;
    const int same = has(t, n_dtype, dtype), here = same == 1 ? on_device(c, t) : same;
    if (same < 0 || here < 0) return -1;
    if (n != 2 || size[0] != rows || size[1] != cols || !same || !here) {
        char what[160];
        PyObject* s = PyObject_Str(dtype);
        PyOS_snprintf(what, sizeof(what), "must be [%lld, %lld] of %s on the device of the first tensor", (long long)rows, (long long)cols,
                      s && PyUnicode_AsUTF8(s) ? PyUnicode_AsUTF8(s) : "?");
        Py_XDECREF(s);
        PyErr_Clear();
        return fail(c, name, what, t);
    }
    PyObject* st = PyObject_CallMethodNoArgs(t, n_stride);
    if (!st) return -1;
    step[0] = PyLong_AsLongLong(PyTuple_GET_ITEM(st, 0));
    step[1] = PyLong_AsLongLong(PyTuple_GET_ITEM(st, 1));
    Py_DECREF(st);
    if (PyErr_Occurred()) return -1;
    if (step[1] != 1 && cols > 1) return fail(c, name, "must have contiguous columns", t);
    if (rows <= 1 && step[0] < cols) step[0] = cols;
    if (step[0] < cols) return fail(c, name, "has rows that overlap", t);
    *ld = step[0];
    return address_of(t, p);
}

/* contiguous array of n elements (n < 0: any number, written to *count; None: a NULL pointer) */
static int flat(const Call* c, PyObject* t, const char* name, int64_t n, PyObject* dtype, void** p, int64_t* count)
{
    *p = NULL;
    if (count) *count = 0;
    if (t == Py_None) return 0;
    int64_t size[4] = {0, 0, 0, 0}, all = 1;
    const int dims = sizes_of(t, size);
    if (dims < 0) return -1;
    for (int i = 0; i < dims && i < 4; ++i) all *= size[i];
    const int same = has(t, n_dtype, dtype), here = same == 1 ? on_device(c, t) : same;
    if (same < 0 || here < 0) return -1;
    PyObject* k = PyObject_CallMethodNoArgs(t, n_is_contiguous);
    if (!k) return -1;
    const int whole = k == Py_True;
    Py_DECREF(k);
    if (dims > 4 || !same || !here || !whole || (n >= 0 && all != n)) {
        char what[160];
        PyObject* s = PyObject_Str(dtype);
        PyOS_snprintf(what, sizeof(what), "must be contiguous %s on the device of the first tensor", s && PyUnicode_AsUTF8(s) ? PyUnicode_AsUTF8(s) : "?");
        if (n >= 0) PyOS_snprintf(what + strlen(what), sizeof(what) - strlen(what), ", %lld elements", (long long)n);
        Py_XDECREF(s);
        PyErr_Clear();
        return fail(c, name, what, t);
    }
    if (count) *count = all;
    return address_of(t, p);
}

static int begin(Call* c, const char* fn, PyObject* first)
{
    c->fn = fn;
    c->device = PyObject_GetAttr(first, n_device);
    return c->device ? 0 : -1;
}

/* the raw stream (the given one's, or the device's current one), and whether the device is the current one: 0, kOtherDevice or -1 */
static int stream_of(Call* c, PyObject* stream, void** raw)
{
    PyObject* type = PyObject_GetAttr(c->device, n_type);
    if (!type) return -1;
    const int cuda = PyUnicode_CompareWithASCIIString(type, "cuda") == 0;
    Py_DECREF(type);
    if (!cuda) {
        PyErr_Format(PyExc_ValueError, "%s: tensors must be on a CUDA device, not %S", c->fn, c->device);
        return -1;
    }
    PyObject* index = PyObject_GetAttr(c->device, n_index);
    if (!index) return -1;
    c->index = index == Py_None ? 0 : PyLong_AsLong(index);
    PyObject* s = NULL;
    if (stream == Py_None) {
        s = PyObject_CallOneArg(c_raw_stream, index);
    } else {
        PyObject* d = PyObject_GetAttr(stream, n_device);
        const int same = d ? PyObject_RichCompareBool(d, c->device, Py_EQ) : -1;
        if (same == 0) PyErr_Format(PyExc_ValueError, "%s: the stream belongs to %S, the tensors to %S", c->fn, d, c->device);
        Py_XDECREF(d);
        if (same == 1) s = PyObject_GetAttr(stream, n_cuda_stream);
    }
    Py_DECREF(index);
    if (!s) return -1;
    *raw = (void*)(uintptr_t)PyLong_AsUnsignedLongLong(s);
    Py_DECREF(s);
    PyObject* now = PyObject_CallNoArgs(c_get_device);
    if (!now) return -1;
    const long cur = PyLong_AsLong(now);
    Py_DECREF(now);
    if (PyErr_Occurred()) return -1;
    return cur == c->index ? 0 : kOtherDevice;
}

static int too_large(const Call* c, int64_t a, int64_t b)
{
    if (a <= INT32_MAX && b <= INT32_MAX) return 0;
    PyErr_Format(PyExc_ValueError, "%s: a dimension does not fit 32 bits", c->fn);
    return 1;
}

/* logits, rule, topk_idx, topk_w, balance_bias, tenant_id, model_of_tenant, tie_flag, status_out, stream */
static PyObject* call_gate(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "moe_gate: 10 arguments"); return NULL; }
    if (begin(&c, "moe_gate", a[0]) < 0) return NULL;
    PyObject* result = NULL;
    Py_buffer rule = {0};
    int64_t zs[4], is[4], bs[4] = {1, 0, 0, 0}, ld, n_tenants;
    void *z, *idx, *w, *bias, *tenant, *mot, *tie, *status, *raw;
    const int zd = sizes_of(a[0], zs), id = zd < 0 ? -1 : sizes_of(a[2], is);
    if (zd < 0 || id < 0) goto done;
    if (zd != 2 || id != 2 || (PyObject*)Py_TYPE(a[1]) != rule_type) {
        PyErr_SetString(PyExc_ValueError, "moe_gate: logits [T, E], a moe_gating() rule and topk_idx [T, k] are needed");
        goto done;
    }
    const int64_t T = zs[0], E = zs[1], k = is[1];
    const int bf16 = has(a[0], n_dtype, t_bf16);
    if (bf16 < 0 || too_large(&c, T, E) || matrix(&c, a[0], "logits", T, E, bf16 ? t_bf16 : t_f32, &z, &ld) < 0) goto done;
    int64_t M = 1;
    if (a[4] != Py_None) {
        const int bd = sizes_of(a[4], bs);
        if (bd < 0) goto done;
        M = bd == 2 ? bs[0] : 1;
    }
    if (flat(&c, a[4], "balance_bias", M * E, t_f32, &bias, NULL) < 0 || flat(&c, a[5], "tenant_id", T, t_i32, &tenant, NULL) < 0 ||
        flat(&c, a[6], "model_of_tenant", -1, t_i32, &mot, &n_tenants) < 0 || flat(&c, a[2], "topk_idx", T * k, t_i32, &idx, NULL) < 0 ||
        flat(&c, a[3], "topk_w", T * k, t_f32, &w, NULL) < 0 || flat(&c, a[7], "tie_flag", T, t_u8, &tie, NULL) < 0 ||
        flat(&c, a[8], "status_out", 1, t_i32, &status, NULL) < 0)
        goto done;
    if (!mot) n_tenants = 1 << 30;
    if (too_large(&c, n_tenants, M)) goto done;
    const int where = stream_of(&c, a[9], &raw);
    if (where < 0 || PyObject_GetBuffer(a[1], &rule, PyBUF_SIMPLE) < 0) goto done;
    const int rc = where ? kOtherDevice
                         : f_gate(z, bf16 ? MOE_TYPE_BF16 : MOE_TYPE_F32, ld, (int)T, (int)E, (int)k, (const moe_gating*)rule.buf, bias, tenant, mot,
                                  (int)n_tenants, (int)M, idx, w, tie, status, raw);
    PyBuffer_Release(&rule);
    result = PyLong_FromLong(rc);
done:
    Py_DECREF(c.device);
    return result;
}

/* x, weight, eps, residual, residual_out, out, out_q, q_scale, stream */
static PyObject* call_norm(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "moe_add_rmsnorm: 9 arguments"); return NULL; }
    if (begin(&c, "moe_add_rmsnorm", a[0]) < 0) return NULL;
    PyObject* result = NULL;
    int64_t xs[4], ss[4], ldx, ldr, ldro, ldo, ldq;
    void *x, *g, *r, *ro, *o, *q, *s, *raw;
    const double eps = PyFloat_AsDouble(a[2]);
    if (eps == -1.0 && PyErr_Occurred()) goto done;
    const int xd = sizes_of(a[0], xs);
    if (xd < 0) goto done;
    if (xd != 2) { fail(&c, "x", "must be [T, H]", a[0]); goto done; }
    const int64_t T = xs[0], H = xs[1];
    if (too_large(&c, T, H) || matrix(&c, a[0], "x", T, H, t_bf16, &x, &ldx) < 0 || flat(&c, a[1], "weight", H, t_bf16, &g, NULL) < 0 ||
        matrix(&c, a[3], "residual", T, H, t_bf16, &r, &ldr) < 0 || matrix(&c, a[4], "residual_out", T, H, t_bf16, &ro, &ldro) < 0 ||
        matrix(&c, a[5], "out", T, H, t_bf16, &o, &ldo) < 0 || matrix(&c, a[6], "out_q", T, H, t_e4m3, &q, &ldq) < 0 ||
        flat(&c, a[7], "q_scale", -1, t_f32, &s, NULL) < 0)
        goto done;
    int group = 0;
    if ((a[6] == Py_None) != (a[7] == Py_None)) { fail(&c, "out_q", "and q_scale go together", NULL); goto done; }
    if (a[7] != Py_None) {
        const int sd = sizes_of(a[7], ss);
        if (sd < 0) goto done;
        if (sd != 2 || ss[0] != T || (ss[1] != 1 && ss[1] != (H + 127) / 128)) { fail(&c, "q_scale", "must be [T, 1] or [T, ceil(H / 128)]", a[7]); goto done; }
        group = ss[1] == 1 ? 0 : 128;            /* (one group of at most 128 columns is the row) */
    }
    const int where = stream_of(&c, a[8], &raw);
    if (where < 0) goto done;
    result = PyLong_FromLong(where ? kOtherDevice : f_norm(x, ldx, r, ldr, g, (float)eps, (int)T, (int)H, ro, ldro, o, ldo, q, ldq, s, group, raw));
done:
    Py_DECREF(c.device);
    return result;
}

/* x, w, out, base, a, b, scale, tenant_id, adapter_of_tenant, n_tenants, workspace, status_out, stream */
static PyObject* call_project(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 13) { PyErr_SetString(PyExc_TypeError, "moe_project: 13 arguments"); return NULL; }
    if (begin(&c, "moe_project", a[0]) < 0) return NULL;
    PyObject *result = NULL, *own = NULL;
    int64_t xs[4], os[4], as[4], bs[4], ldx, ldw, ldo, ldb, ws_bytes = 0, n_tenants = 0;
    void *x, *w, *o, *base, *pa = NULL, *pb = NULL, *scale = NULL, *tenant = NULL, *table = NULL, *ws = NULL, *status, *raw;
    const int xd = sizes_of(a[0], xs), od = xd < 0 ? -1 : sizes_of(a[2], os);
    if (xd < 0 || od < 0) goto done;
    if (xd != 2 || od != 2) { fail(&c, "x", "must be [T, K] and out [T, N]", a[0]); goto done; }
    const int64_t T = xs[0], K = xs[1], N = os[1];
    const int f32 = has(a[2], n_dtype, t_f32);
    PyObject* ot = f32 == 1 ? t_f32 : t_bf16;
    if (f32 < 0 || too_large(&c, T, K) || too_large(&c, N, N) || matrix(&c, a[0], "x", T, K, t_bf16, &x, &ldx) < 0 ||
        matrix(&c, a[1], "w", N, K, t_bf16, &w, &ldw) < 0 || matrix(&c, a[2], "out", T, N, ot, &o, &ldo) < 0 ||
        matrix(&c, a[3], "base", T, N, ot, &base, &ldb) < 0)
        goto done;
    int64_t adapters = 0, rank = 0;
    if ((a[4] == Py_None) != (a[5] == Py_None)) { fail(&c, "a", "and b go together", NULL); goto done; }
    if (a[4] != Py_None) {
        const int ad = sizes_of(a[4], as), bd = ad < 0 ? -1 : sizes_of(a[5], bs);
        if (ad < 0 || bd < 0) goto done;
        if (ad != 3 || as[2] != K) { fail(&c, "a", "must be [n_adapters, rank, K]", a[4]); goto done; }
        adapters = as[0]; rank = as[1];
        if (bd != 3 || bs[0] != adapters || bs[1] != N || bs[2] != rank) { fail(&c, "b", "must be [n_adapters, N, rank]", a[5]); goto done; }
        if (too_large(&c, adapters, rank) || flat(&c, a[4], "a", -1, t_bf16, &pa, NULL) < 0 || flat(&c, a[5], "b", -1, t_bf16, &pb, NULL) < 0 ||
            flat(&c, a[6], "scale", adapters, t_f32, &scale, NULL) < 0 || flat(&c, a[7], "tenant_id", T, t_i32, &tenant, NULL) < 0 ||
            flat(&c, a[8], "adapter_of_tenant", -1, t_i32, &table, &n_tenants) < 0)
            goto done;
        if (a[8] == Py_None) n_tenants = a[9] == Py_None ? adapters : PyLong_AsLongLong(a[9]);
        if (PyErr_Occurred() || too_large(&c, n_tenants, 0)) goto done;
    }
    if (flat(&c, a[10], "workspace", -1, t_u8, &ws, &ws_bytes) < 0 || flat(&c, a[11], "status_out", 1, t_i32, &status, NULL) < 0) goto done;
    const int where = stream_of(&c, a[12], &raw);
    if (where < 0) goto done;
    if (where) { result = PyLong_FromLong(kOtherDevice); goto done; }
    if (a[10] == Py_None) {
        const int64_t need = f_workspace((int)T, (int)K, (int)N, (int)rank, (int)adapters);
        if (need > 0) {                          /* (allocated on the stream of the call: the current one) */
            own = PyObject_CallFunction(c_empty, "LO", (long long)need, c.device);
            if (!own || address_of(own, &ws) < 0) goto done;
            ws_bytes = need;
        }
    }
    result = PyLong_FromLong(f_project(x, ldx, w, ldw, (int)T, (int)K, (int)N, pa, pb, scale, (int)adapters, (int)rank, tenant, table, (int)n_tenants,
                                       base, ldb, o, ldo, f32 ? MOE_TYPE_F32 : MOE_TYPE_BF16, ws, ws_bytes, status, raw));
done:
    Py_XDECREF(own);
    Py_DECREF(c.device);
    return result;
}

/* a call's own workspace, allocated on its stream (the current one) where the caller gave none: 0 or -1 */
static int own_workspace(const Call* c, int64_t need, PyObject** own, void** ws, int64_t* bytes)
{
    if (need <= 0) return 0;
    *own = PyObject_CallFunction(c_empty, "LO", (long long)need, c->device);
    if (!*own || address_of(*own, ws) < 0) return -1;
    *bytes = need;
    return 0;
}

/* a block's gate: None, float32 [T], bf16 [H] or bf16 [T, H]; into *rule and *gate */
static int gate_of(const Call* c, PyObject* t, PyObject* act, int64_t T, int64_t H, moe_block_rule* rule, void** gate, int64_t* ld)
{
    *gate = NULL; *ld = 0;
    rule->gate = MOE_GATE_NONE;
    rule->gate_act = (int32_t)PyLong_AsLong(act);
    if (PyErr_Occurred()) return -1;
    if (t == Py_None) return 0;
    int64_t size[4];
    const int dims = sizes_of(t, size), f32 = dims < 0 ? -1 : has(t, n_dtype, t_f32);
    if (f32 < 0) return -1;
    rule->gate = f32 ? MOE_GATE_TOKEN : dims == 1 ? MOE_GATE_CHANNEL : MOE_GATE_ELEMENT;
    if (rule->gate == MOE_GATE_ELEMENT) return matrix(c, t, "gate", T, H, t_bf16, gate, ld);
    return flat(c, t, "gate", f32 ? T : H, f32 ? t_f32 : t_bf16, gate, NULL);
}

static int floats(PyObject* const* a, float* v, int n)
{
    for (int i = 0; i < n; ++i) v[i] = (float)PyFloat_AsDouble(a[i]);
    return PyErr_Occurred() ? -1 : 0;
}

/* block_out, residual, h, eps, post_weight, pre_weight, gate, gate_act, residual_scale, block_scale, out, out_q, q_scale, stream */
static PyObject* call_block(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 14) { PyErr_SetString(PyExc_TypeError, "moe_block_norm: 14 arguments"); return NULL; }
    if (begin(&c, "moe_block_norm", a[0]) < 0) return NULL;
    PyObject* result = NULL;
    int64_t s[4], ldy, ldr, ldh, ldg, ldo, ldq;
    void *y, *r, *h, *post, *pre, *gate, *o, *q, *qs, *raw;
    moe_block_rule rule;
    const int d = sizes_of(a[0], s);
    if (d < 0 || floats(a + 3, &rule.eps, 1) < 0 || floats(a + 8, &rule.residual_scale, 1) < 0 || floats(a + 9, &rule.block_scale, 1) < 0) goto done;
    if (d != 2) { fail(&c, "block_out", "must be [T, H]", a[0]); goto done; }
    const int64_t T = s[0], H = s[1];
    if (a[1] == Py_None || a[2] == Py_None) { fail(&c, "residual", "and h are needed", NULL); goto done; }
    if ((a[11] == Py_None) != (a[12] == Py_None)) { fail(&c, "out_q", "and q_scale go together", NULL); goto done; }
    if (too_large(&c, T, H) || matrix(&c, a[0], "block_out", T, H, t_bf16, &y, &ldy) < 0 || matrix(&c, a[1], "residual", T, H, t_bf16, &r, &ldr) < 0 ||
        matrix(&c, a[2], "h", T, H, t_bf16, &h, &ldh) < 0 || flat(&c, a[4], "post_weight", H, t_bf16, &post, NULL) < 0 ||
        flat(&c, a[5], "pre_weight", H, t_bf16, &pre, NULL) < 0 || gate_of(&c, a[6], a[7], T, H, &rule, &gate, &ldg) < 0 ||
        matrix(&c, a[10], "out", T, H, t_bf16, &o, &ldo) < 0 || matrix(&c, a[11], "out_q", T, H, t_i8, &q, &ldq) < 0 ||
        flat(&c, a[12], "q_scale", T, t_f32, &qs, NULL) < 0)
        goto done;
    const int where = stream_of(&c, a[13], &raw);
    if (where < 0) goto done;
    result = PyLong_FromLong(where ? kOtherDevice
                                   : f_block(y, ldy, r, ldr, post, pre, gate, ldg, &rule, (int)T, (int)H, h, ldh, o, ldo, q, ldq, qs, raw));
done:
    Py_DECREF(c.device);
    return result;
}

/* block_out, h, eps, post_weight, pre_weight, gate, gate_act, residual_scale, block_scale, d_out, d_h, d_block, d_residual, d_gate,
 * d_post_weight, d_pre_weight, workspace, stream */
static PyObject* call_block_grad(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 18) { PyErr_SetString(PyExc_TypeError, "moe_block_norm_backward: 18 arguments"); return NULL; }
    if (begin(&c, "moe_block_norm_backward", a[0]) < 0) return NULL;
    PyObject *result = NULL, *own = NULL;
    int64_t s[4], ldy, ldh, ldg, ldo, ldd, ldb, ldr, ldgg = 0, ws_bytes = 0;
    void *y, *h, *post, *pre, *gate, *d_out, *d_h, *d_block, *d_res, *d_gate = NULL, *d_post, *d_pre, *ws, *raw;
    moe_block_rule rule;
    const int d = sizes_of(a[0], s);
    if (d < 0 || floats(a + 2, &rule.eps, 1) < 0 || floats(a + 7, &rule.residual_scale, 1) < 0 || floats(a + 8, &rule.block_scale, 1) < 0) goto done;
    if (d != 2) { fail(&c, "block_out", "must be [T, H]", a[0]); goto done; }
    const int64_t T = s[0], H = s[1];
    if (too_large(&c, T, H) || matrix(&c, a[0], "block_out", T, H, t_bf16, &y, &ldy) < 0 || matrix(&c, a[1], "h", T, H, t_bf16, &h, &ldh) < 0 ||
        flat(&c, a[3], "post_weight", H, t_bf16, &post, NULL) < 0 || flat(&c, a[4], "pre_weight", H, t_bf16, &pre, NULL) < 0 ||
        gate_of(&c, a[5], a[6], T, H, &rule, &gate, &ldg) < 0 || matrix(&c, a[9], "d_out", T, H, t_bf16, &d_out, &ldo) < 0 ||
        matrix(&c, a[10], "d_h", T, H, t_bf16, &d_h, &ldd) < 0 || matrix(&c, a[11], "d_block", T, H, t_bf16, &d_block, &ldb) < 0 ||
        matrix(&c, a[12], "d_residual", T, H, t_bf16, &d_res, &ldr) < 0 || flat(&c, a[14], "d_post_weight", H, t_f32, &d_post, NULL) < 0 ||
        flat(&c, a[15], "d_pre_weight", H, t_f32, &d_pre, NULL) < 0 || flat(&c, a[16], "workspace", -1, t_u8, &ws, &ws_bytes) < 0)
        goto done;
    if (a[13] != Py_None) {
        if (rule.gate == MOE_GATE_NONE) { fail(&c, "d_gate", "needs a gate", NULL); goto done; }
        if ((rule.gate == MOE_GATE_ELEMENT ? matrix(&c, a[13], "d_gate", T, H, t_bf16, &d_gate, &ldgg)
                                           : flat(&c, a[13], "d_gate", rule.gate == MOE_GATE_TOKEN ? T : H, t_f32, &d_gate, NULL)) < 0)
            goto done;
    }
    const int where = stream_of(&c, a[17], &raw);
    if (where < 0) goto done;
    if (where) { result = PyLong_FromLong(kOtherDevice); goto done; }
    if (a[16] == Py_None && T > 0 && (d_post || d_pre || (d_gate && rule.gate == MOE_GATE_CHANNEL)) &&
        own_workspace(&c, f_block_workspace((int)T, (int)H), &own, &ws, &ws_bytes) < 0)
        goto done;
    result = PyLong_FromLong(f_block_grad(y, ldy, h, ldh, post, pre, gate, ldg, &rule, (int)T, (int)H, d_out, ldo, d_h, ldd, d_block, ldb, d_res, ldr,
                                          d_gate, ldgg, d_post, d_pre, ws, ws_bytes, raw));
done:
    Py_XDECREF(own);
    Py_DECREF(c.device);
    return result;
}

/* x, q, scale, stream */
static PyObject* call_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "moe_quantize_i8: 4 arguments"); return NULL; }
    if (begin(&c, "moe_quantize_i8", a[0]) < 0) return NULL;
    PyObject* result = NULL;
    int64_t s[4], ldx, ldq;
    void *x, *q, *scale, *raw;
    const int d = sizes_of(a[0], s);
    if (d < 0) goto done;
    if (d != 2) { fail(&c, "x", "must be [T, K]", a[0]); goto done; }
    if (a[1] == Py_None || a[2] == Py_None) { fail(&c, "q", "and scale are needed", NULL); goto done; }
    if (too_large(&c, s[0], s[1]) || matrix(&c, a[0], "x", s[0], s[1], t_bf16, &x, &ldx) < 0 || matrix(&c, a[1], "q", s[0], s[1], t_i8, &q, &ldq) < 0 ||
        flat(&c, a[2], "scale", s[0], t_f32, &scale, NULL) < 0)
        goto done;
    const int where = stream_of(&c, a[3], &raw);
    if (where < 0) goto done;
    result = PyLong_FromLong(where ? kOtherDevice : f_quantize(x, ldx, (int)s[0], (int)s[1], q, ldq, scale, raw));
done:
    Py_DECREF(c.device);
    return result;
}

/* x, x_scale, w, w_scale, out, bias, base, status_out, stream */
static PyObject* call_project_i8(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "moe_project_i8: 9 arguments"); return NULL; }
    if (begin(&c, "moe_project_i8", a[0]) < 0) return NULL;
    PyObject* result = NULL;
    int64_t xs[4], os[4], ldx, ldw, ldo, ldb;
    void *x, *xscale, *w, *wscale, *o, *bias, *base, *status, *raw;
    const int xd = sizes_of(a[0], xs), od = xd < 0 ? -1 : sizes_of(a[4], os);
    if (xd < 0 || od < 0) goto done;
    if (xd != 2 || od != 2) { fail(&c, "x", "must be [T, K] and out [T, N]", a[0]); goto done; }
    if (a[1] == Py_None || a[2] == Py_None || a[3] == Py_None) { fail(&c, "x_scale", ", w and w_scale are needed", NULL); goto done; }
    const int64_t T = xs[0], K = xs[1], N = os[1];
    const int f32 = has(a[4], n_dtype, t_f32);
    PyObject* ot = f32 == 1 ? t_f32 : t_bf16;
    if (f32 < 0 || too_large(&c, T, K) || too_large(&c, N, N) || matrix(&c, a[0], "x", T, K, t_i8, &x, &ldx) < 0 ||
        flat(&c, a[1], "x_scale", T, t_f32, &xscale, NULL) < 0 || matrix(&c, a[2], "w", N, K, t_i8, &w, &ldw) < 0 ||
        flat(&c, a[3], "w_scale", N, t_f32, &wscale, NULL) < 0 || matrix(&c, a[4], "out", T, N, ot, &o, &ldo) < 0 ||
        flat(&c, a[5], "bias", N, t_f32, &bias, NULL) < 0 || matrix(&c, a[6], "base", T, N, ot, &base, &ldb) < 0 ||
        flat(&c, a[7], "status_out", 1, t_i32, &status, NULL) < 0)
        goto done;
    /* (a single row's distance is that of its neighbours-to-be: any) */
    if (T <= 1) ldx = (ldx + 15) / 16 * 16;
    if (N <= 1) ldw = (ldw + 15) / 16 * 16;
    const int where = stream_of(&c, a[8], &raw);
    if (where < 0) goto done;
    result = PyLong_FromLong(where ? kOtherDevice
                                   : f_project_i8(x, ldx, xscale, w, ldw, wscale, (int)T, (int)K, (int)N, bias, base, ldb, o, ldo,
                                                  f32 ? MOE_TYPE_F32 : MOE_TYPE_BF16, status, raw));
done:
    Py_DECREF(c.device);
    return result;
}

/* what a router's training reads, out of logits, topk_idx, mask, tenant_id, model_of_tenant */
typedef struct {
    int64_t T, E, k, ld, n_tenants;
    int bf16;
    void *z, *idx, *mask, *tenant, *mot;
} Router;
static int router_of(const Call* c, PyObject* logits, PyObject* idx, PyObject* mask, PyObject* tenant, PyObject* mot, Router* r)
{
    int64_t zs[4], is[4];
    const int zd = sizes_of(logits, zs), id = zd < 0 ? -1 : sizes_of(idx, is);
    if (zd < 0 || id < 0) return -1;
    if (zd != 2 || id != 2) return fail(c, "logits", "must be [T, E] and topk_idx [T, k]", logits);
    r->T = zs[0]; r->E = zs[1]; r->k = is[1];
    r->bf16 = has(logits, n_dtype, t_bf16);
    if (r->bf16 < 0 || too_large(c, r->T, r->E) || too_large(c, r->k, r->k) ||
        matrix(c, logits, "logits", r->T, r->E, r->bf16 ? t_bf16 : t_f32, &r->z, &r->ld) < 0 ||
        flat(c, idx, "topk_idx", r->T * r->k, t_i32, &r->idx, NULL) < 0 || flat(c, mask, "mask", r->T, t_u8, &r->mask, NULL) < 0 ||
        flat(c, tenant, "tenant_id", r->T, t_i32, &r->tenant, NULL) < 0 || flat(c, mot, "model_of_tenant", -1, t_i32, &r->mot, &r->n_tenants) < 0)
        return -1;
    if (!r->mot) r->n_tenants = 1 << 30;
    return too_large(c, r->n_tenants, 0) ? -1 : 0;
}

/* logits, topk_idx, counts, tokens, mean_prob, loss, score, z_loss, mask, tenant_id, model_of_tenant, workspace, status_out, stream */
static PyObject* call_balance(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 14) { PyErr_SetString(PyExc_TypeError, "moe_balance_loss: 14 arguments"); return NULL; }
    if (begin(&c, "moe_balance_loss", a[0]) < 0) return NULL;
    PyObject *result = NULL, *own = NULL;
    Router r;
    int64_t cs[4], ws_bytes = 0;
    void *counts, *tokens, *mean, *loss, *z, *ws, *status, *raw;
    const long score = PyLong_AsLong(a[6]);
    if (PyErr_Occurred() || router_of(&c, a[0], a[1], a[8], a[9], a[10], &r) < 0) goto done;
    if (a[2] == Py_None || a[3] == Py_None || a[4] == Py_None || a[5] == Py_None) { fail(&c, "counts", ", tokens, mean_prob and loss are needed", NULL); goto done; }
    const int cd = sizes_of(a[2], cs);
    if (cd < 0) goto done;
    const int64_t M = cd == 2 ? cs[0] : 1;                   /* (counts of one model may be [E]) */
    if (too_large(&c, M, 0) || flat(&c, a[2], "counts", M * r.E, t_i32, &counts, NULL) < 0 || flat(&c, a[3], "tokens", M, t_i32, &tokens, NULL) < 0 ||
        flat(&c, a[4], "mean_prob", M * r.E, t_f32, &mean, NULL) < 0 || flat(&c, a[5], "loss", M, t_f32, &loss, NULL) < 0 ||
        flat(&c, a[7], "z_loss", M, t_f32, &z, NULL) < 0 || flat(&c, a[11], "workspace", -1, t_u8, &ws, &ws_bytes) < 0 ||
        flat(&c, a[12], "status_out", 1, t_i32, &status, NULL) < 0)
        goto done;
    const int where = stream_of(&c, a[13], &raw);
    if (where < 0) goto done;
    if (where) { result = PyLong_FromLong(kOtherDevice); goto done; }
    if (a[11] == Py_None && own_workspace(&c, f_balance_workspace((int)r.T, (int)r.E, (int)M), &own, &ws, &ws_bytes) < 0) goto done;
    result = PyLong_FromLong(f_balance(r.z, r.bf16 ? MOE_TYPE_BF16 : MOE_TYPE_F32, r.ld, (int)r.T, (int)r.E, (int)r.k, (int)score, r.idx, r.mask, r.tenant,
                                       r.mot, (int)r.n_tenants, (int)M, counts, tokens, mean, loss, z, ws, ws_bytes, status, raw));
done:
    Py_XDECREF(own);
    Py_DECREF(c.device);
    return result;
}

/* logits, rule, topk_idx, d_logits, d_topk_w, counts, tokens, d_loss, d_z_loss, mask, tenant_id, model_of_tenant, status_out, stream */
static PyObject* call_gate_grad(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Call c;
    if (n != 14) { PyErr_SetString(PyExc_TypeError, "moe_gate_backward: 14 arguments"); return NULL; }
    if (begin(&c, "moe_gate_backward", a[0]) < 0) return NULL;
    PyObject* result = NULL;
    Py_buffer rule = {0};
    Router r;
    int64_t ldd, M = 1, count;
    void *d, *dw, *counts, *tokens, *dl, *dz, *status, *raw;
    if ((PyObject*)Py_TYPE(a[1]) != rule_type) { PyErr_SetString(PyExc_ValueError, "moe_gate_backward: a moe_gating() rule is needed"); goto done; }
    if (router_of(&c, a[0], a[2], a[9], a[10], a[11], &r) < 0) goto done;
    if (a[3] == Py_None) { fail(&c, "d_logits", "is needed", NULL); goto done; }
    if (matrix(&c, a[3], "d_logits", r.T, r.E, r.bf16 ? t_bf16 : t_f32, &d, &ldd) < 0 || flat(&c, a[4], "d_topk_w", r.T * r.k, t_f32, &dw, NULL) < 0 ||
        flat(&c, a[7], "d_loss", -1, t_f32, &dl, &count) < 0)
        goto done;
    /* the number of models is that of the losses */
    if (dl) M = count;
    if (flat(&c, a[8], "d_z_loss", dl ? M : -1, t_f32, &dz, &count) < 0) goto done;
    if (!dl && dz) M = count;
    if (too_large(&c, M, 0) || flat(&c, a[5], "counts", dl ? M * r.E : -1, t_i32, &counts, NULL) < 0 ||
        flat(&c, a[6], "tokens", dl || dz ? M : -1, t_i32, &tokens, NULL) < 0 || flat(&c, a[12], "status_out", 1, t_i32, &status, NULL) < 0)
        goto done;
    const int where = stream_of(&c, a[13], &raw);
    if (where < 0 || PyObject_GetBuffer(a[1], &rule, PyBUF_SIMPLE) < 0) goto done;
    const int rc = where ? kOtherDevice
                         : f_gate_grad(r.z, r.bf16 ? MOE_TYPE_BF16 : MOE_TYPE_F32, r.ld, (int)r.T, (int)r.E, (int)r.k, (const moe_gating*)rule.buf, r.idx,
                                       dw, r.mask, r.tenant, r.mot, (int)r.n_tenants, (int)M, counts, tokens, dl, dz, d, ldd, status, raw);
    PyBuffer_Release(&rule);
    result = PyLong_FromLong(rc);
done:
    Py_DECREF(c.device);
    return result;
}

/* bind(addresses of moe_gate, moe_add_rmsnorm, moe_project, moe_project_workspace, moe_block_norm, moe_block_norm_backward,
 *      moe_block_norm_workspace, moe_quantize_i8, moe_project_i8, moe_balance_loss, moe_balance_workspace, moe_gate_backward; float32,
 *      bfloat16, int32, uint8, float8_e4m3fn, int8; raw_stream(index), get_device(), empty(bytes, device), class of the gating struct) */
static PyObject* bind(PyObject* self, PyObject* args)
{
    unsigned long long f[12];
    PyObject** keep[] = {&t_f32, &t_bf16, &t_i32, &t_u8, &t_e4m3, &t_i8, &c_raw_stream, &c_get_device, &c_empty, &rule_type};
    PyObject* v[10];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKOOOOOOOOOO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8], &f[9], &f[10], &f[11], &v[0],
                          &v[1], &v[2], &v[3], &v[4], &v[5], &v[6], &v[7], &v[8], &v[9]))
        return NULL;
    f_gate = (gate_fn)(uintptr_t)f[0]; f_norm = (norm_fn)(uintptr_t)f[1]; f_project = (project_fn)(uintptr_t)f[2];
    f_workspace = (workspace_fn)(uintptr_t)f[3]; f_block = (block_fn)(uintptr_t)f[4]; f_block_grad = (block_grad_fn)(uintptr_t)f[5];
    f_block_workspace = (block_workspace_fn)(uintptr_t)f[6]; f_quantize = (quantize_fn)(uintptr_t)f[7];
    f_project_i8 = (project_i8_fn)(uintptr_t)f[8]; f_balance = (balance_fn)(uintptr_t)f[9];
    f_balance_workspace = (balance_workspace_fn)(uintptr_t)f[10]; f_gate_grad = (gate_grad_fn)(uintptr_t)f[11];
    for (int i = 0; i < 10; ++i) { Py_INCREF(v[i]); Py_XSETREF(*keep[i], v[i]); }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "hands over the entry points and torch's objects"},
    {"moe_gate", (PyCFunction)(void (*)(void))call_gate, METH_FASTCALL, "see binding.moe_gate"},
    {"moe_add_rmsnorm", (PyCFunction)(void (*)(void))call_norm, METH_FASTCALL, "see binding.moe_add_rmsnorm"},
    {"moe_project", (PyCFunction)(void (*)(void))call_project, METH_FASTCALL, "see binding.moe_project"},
    {"moe_block_norm", (PyCFunction)(void (*)(void))call_block, METH_FASTCALL, "see binding.moe_block_norm"},
    {"moe_block_norm_backward", (PyCFunction)(void (*)(void))call_block_grad, METH_FASTCALL, "see binding.moe_block_norm_backward"},
    {"moe_quantize_i8", (PyCFunction)(void (*)(void))call_quantize, METH_FASTCALL, "see binding.moe_quantize_i8"},
    {"moe_project_i8", (PyCFunction)(void (*)(void))call_project_i8, METH_FASTCALL, "see binding.moe_project_i8"},
    {"moe_balance_loss", (PyCFunction)(void (*)(void))call_balance, METH_FASTCALL, "see binding.moe_balance_loss"},
    {"moe_gate_backward", (PyCFunction)(void (*)(void))call_gate_grad, METH_FASTCALL, "see binding.moe_gate_backward"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "marshalling of the entry points that take no context", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void)
{
    n_dtype = PyUnicode_InternFromString("dtype"); n_device = PyUnicode_InternFromString("device");
    n_shape = PyUnicode_InternFromString("shape"); n_stride = PyUnicode_InternFromString("stride");
    n_data_ptr = PyUnicode_InternFromString("data_ptr"); n_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    n_type = PyUnicode_InternFromString("type"); n_index = PyUnicode_InternFromString("index");
    n_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return PyModule_Create(&module);
}
