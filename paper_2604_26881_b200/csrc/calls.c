/* Python front-end of the entry points that take no context (moe_gate, moe_add_rmsnorm, moe_project).
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

static gate_fn f_gate;
static norm_fn f_norm;
static project_fn f_project;
static workspace_fn f_workspace;
static PyObject *t_f32, *t_bf16, *t_i32, *t_u8, *t_e4m3;                 /* torch dtypes */
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

/* bind(addresses of moe_gate, moe_add_rmsnorm, moe_project, moe_project_workspace; float32, bfloat16, int32, uint8, float8_e4m3fn;
 *      raw_stream(index), get_device(), empty(bytes, device), class of the gating struct) */
static PyObject* bind(PyObject* self, PyObject* args)
{
    unsigned long long g, m, p, w;
    PyObject** keep[] = {&t_f32, &t_bf16, &t_i32, &t_u8, &t_e4m3, &c_raw_stream, &c_get_device, &c_empty, &rule_type};
    PyObject* v[9];
    if (!PyArg_ParseTuple(args, "KKKKOOOOOOOOO", &g, &m, &p, &w, &v[0], &v[1], &v[2], &v[3], &v[4], &v[5], &v[6], &v[7], &v[8])) return NULL;
    f_gate = (gate_fn)(uintptr_t)g; f_norm = (norm_fn)(uintptr_t)m; f_project = (project_fn)(uintptr_t)p; f_workspace = (workspace_fn)(uintptr_t)w;
    for (int i = 0; i < 9; ++i) { Py_INCREF(v[i]); Py_XSETREF(*keep[i], v[i]); }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "hands over the entry points and torch's objects"},
    {"moe_gate", (PyCFunction)(void (*)(void))call_gate, METH_FASTCALL, "see binding.moe_gate"},
    {"moe_add_rmsnorm", (PyCFunction)(void (*)(void))call_norm, METH_FASTCALL, "see binding.moe_add_rmsnorm"},
    {"moe_project", (PyCFunction)(void (*)(void))call_project, METH_FASTCALL, "see binding.moe_project"},
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
