/* Argument marshalling of the asynchronous calls for the Python binding.  These calls only
 * enqueue a few microseconds of GPU work, so what the interpreter spends on describing them is
 * part of their cost: through ctypes (a Structure built per call, seven converted arguments) and
 * a torch.cuda.Stream object about 5 us a call, here about 2 (4096 rows of 16, one
 * seer_spmv_auto 12.3 -> 9.2 us; 19 prepared products of 2.5 M nonzeros 174 -> 93 us).
 * Everything is read from the objects anew on every call; nothing is kept.  The library's
 * functions are handed over as addresses (bind), so the module links against nothing. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/seer.h"

static int (*f_spmv)(int, const seer_csr *, const float *, float *, void *, size_t, void *);
static int (*f_auto)(const seer_csr *, const seer_tree *, const float *, float *, void *, size_t, void *);
static int (*f_model)(const seer_csr *, const seer_model *, const float *, float *, void *, size_t, void *, int *, int *);
static int (*f_prepared)(const seer_plan *, const seer_csr *, const float *, float *, void *, size_t, void *);

static PyObject *s_rows, *s_cols, *s_nnz, *s_row_ptr, *s_col_idx, *s_values, *s_data_ptr, *s_numel;

/* What ctypes takes: for a size anything that is an integer (None and floats raise TypeError),
 * reduced to the width of the parameter; for an address an int, or None for a null pointer. */
static int as_size(PyObject *o, uint64_t *out)
{
    *out = (uint64_t)PyLong_AsUnsignedLongLongMask(o);
    return PyErr_Occurred() ? -1 : 0;
}

static int as_address(PyObject *o, uint64_t *out)
{
    if (o == Py_None) { *out = 0; return 0; }
    if (!PyLong_Check(o)) {
        PyErr_Format(PyExc_TypeError, "an address must be an int, not %.100s", Py_TYPE(o)->tp_name);
        return -1;
    }
    return as_size(o, out);
}

/* Takes over the reference r (null: an exception is set). */
static int taken(PyObject *r, int (*as)(PyObject *, uint64_t *), uint64_t *out)
{
    if (!r) return -1;
    const int rc = as(r, out);
    Py_DECREF(r);
    return rc;
}

static int size_attr(PyObject *o, PyObject *name, uint64_t *out) { return taken(PyObject_GetAttr(o, name), as_size, out); }

static int address_of(PyObject *tensor, uint64_t *out)
{
    return taken(PyObject_CallMethodNoArgs(tensor, s_data_ptr), as_address, out);
}

static int address_attr(PyObject *o, PyObject *name, uint64_t *out)
{
    PyObject *t = PyObject_GetAttr(o, name);
    if (!t) return -1;
    const int rc = address_of(t, out);
    Py_DECREF(t);
    return rc;
}

/* DeviceCSR.c_struct() */
static int csr_of(PyObject *A, seer_csr *c)
{
    uint64_t rows, cols, nnz, rp, ci = 0, va = 0;
    if (size_attr(A, s_rows, &rows) || size_attr(A, s_cols, &cols) || size_attr(A, s_nnz, &nnz) ||
        address_attr(A, s_row_ptr, &rp))
        return -1;
    if (nnz && (address_attr(A, s_col_idx, &ci) || address_attr(A, s_values, &va))) return -1;
    c->rows = (int32_t)rows;
    c->cols = (int32_t)cols;
    c->nnz = (int32_t)nnz;
    c->row_ptr = (const int32_t *)(uintptr_t)rp;
    c->col_idx = (const int32_t *)(uintptr_t)ci;
    c->values = (const float *)(uintptr_t)va;
    return 0;
}

/* x, y, workspace (may be None) and the stream handle: arguments 2 .. 5 of every call below */
typedef struct {
    seer_csr csr;
    uint64_t handle, x, y, ws, ws_bytes, stream;
} call_args;

static int parse(PyObject *const *a, Py_ssize_t n, call_args *c)
{
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "expected (handle, matrix, x, y, workspace, stream)");
        return -1;
    }
    c->ws = c->ws_bytes = 0;
    if (as_size(a[0], &c->handle) || csr_of(a[1], &c->csr) || address_of(a[2], &c->x) || address_of(a[3], &c->y)) return -1;
    if (a[4] != Py_None &&
        (address_of(a[4], &c->ws) || taken(PyObject_CallMethodNoArgs(a[4], s_numel), as_size, &c->ws_bytes)))
        return -1;
    return as_size(a[5], &c->stream);
}

#define P(T, v) ((T)(uintptr_t)(v))

static PyObject *m_spmv(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    call_args c;
    int rc;
    if (parse(a, n, &c)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = f_spmv((int)c.handle, &c.csr, P(const float *, c.x), P(float *, c.y), P(void *, c.ws), (size_t)c.ws_bytes,
                P(void *, c.stream));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *m_auto(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    call_args c;
    int rc;
    if (parse(a, n, &c)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = f_auto(&c.csr, P(const seer_tree *, c.handle), P(const float *, c.x), P(float *, c.y), P(void *, c.ws),
                (size_t)c.ws_bytes, P(void *, c.stream));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *m_model(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    call_args c;
    int rc, path = -1, kid = -1;
    if (parse(a, n, &c)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = f_model(&c.csr, P(const seer_model *, c.handle), P(const float *, c.x), P(float *, c.y), P(void *, c.ws),
                 (size_t)c.ws_bytes, P(void *, c.stream), &path, &kid);
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iii)", rc, path, kid);
}

static PyObject *m_prepared(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    call_args c;
    int rc;
    if (parse(a, n, &c)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = f_prepared(P(const seer_plan *, c.handle), &c.csr, P(const float *, c.x), P(float *, c.y), P(void *, c.ws),
                    (size_t)c.ws_bytes, P(void *, c.stream));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *m_bind(PyObject *self, PyObject *args)
{
    unsigned long long spmv, autos, model, prepared;
    if (!PyArg_ParseTuple(args, "KKKK", &spmv, &autos, &model, &prepared)) return NULL;
    f_spmv = P(int (*)(int, const seer_csr *, const float *, float *, void *, size_t, void *), spmv);
    f_auto = P(int (*)(const seer_csr *, const seer_tree *, const float *, float *, void *, size_t, void *), autos);
    f_model = P(int (*)(const seer_csr *, const seer_model *, const float *, float *, void *, size_t, void *, int *, int *), model);
    f_prepared = P(int (*)(const seer_plan *, const seer_csr *, const float *, float *, void *, size_t, void *), prepared);
    Py_RETURN_NONE;
}

/* ---- the routed layer (routed.py): tensors are described from their own attributes */

static int (*f_route)(const void *, int32_t, const seer_routing *, void *, size_t, void *);
static int (*f_gather)(const seer_routing *, const seer_dense *, const float *, const seer_dense *, void *);
static int (*f_combine)(const seer_routing *, const seer_dense *, const float *, const seer_dense *, void *);
static int (*f_grad)(const seer_routing *, const seer_dense *, const seer_dense *, const float *, const seer_dense *, float *, void *);
static int (*f_quantize)(const seer_dense *, const seer_dense *, float *, void *);
static int (*f_gather_i8)(const seer_routing *, const seer_dense *, const seer_dense *, float *, void *);
static int (*f_product)(const seer_dense *, const float *, const seer_dense *, const float *, const int32_t *, int32_t,
                        const seer_dense *, void *, size_t, void *);
static int (*f_norm)(const seer_grad *, int32_t, float *, void *, size_t, void *);
static int (*f_clip)(const seer_grad *, int32_t, float, float *, void *, size_t, void *);

static PyObject *s_shape, *s_stride, *s_dtype, *s_get_device, *s_initialized, *s_get_current, *s_requires_grad, *s_is_contiguous, *s_tokens, *s_choices, *s_experts, *s_expert_ptr,
    *s_slot_choice, *s_choice_slot, *s_nbytes;
static PyObject *types[6];                   /* torch's dtypes in the order of seer_type */
static PyObject *t_c, *t_cuda;               /* torch._C and torch.cuda, which know the current GPU */
static PyObject *grad_enabled;               /* what says whether torch records a history */

static int refuse(PyObject *error, const char *what, const char *is)
{
    PyErr_Format(error, "%s %s", what, is);
    return -1;
}

/* Truth of what a method returns. */
static int truth(PyObject *t, PyObject *name)
{
    PyObject *v = PyObject_CallMethodNoArgs(t, name);
    if (!v) return -1;
    const int is = PyObject_IsTrue(v);
    Py_DECREF(v);
    return is;
}

static int type_of(PyObject *t, const char *what)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    for (int i = 0; i < 6; ++i)
        if (d == types[i]) {
            Py_DECREF(d);
            return i;
        }
    PyErr_Format(PyExc_TypeError, "%s is %S", what, d);
    Py_DECREF(d);
    return -1;
}

/* The entries of a tuple of at most 3 integers; how many, or -1. */
static int numbers(PyObject *tuple, int64_t out[3])
{
    if (!tuple) return -1;
    int n = -1;
    if (PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) <= 3) {
        n = (int)PyTuple_GET_SIZE(tuple);
        for (int i = 0; i < n; ++i) out[i] = (int64_t)PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
        if (PyErr_Occurred()) n = -1;
    } else n = 4;
    Py_DECREF(tuple);
    return n;
}

/* The GPU that a tensor is on (-1: none), or -2. */
static int gpu_of(PyObject *t)
{
    uint64_t n;
    if (taken(PyObject_CallMethodNoArgs(t, s_get_device), as_size, &n)) return -2;
    return (int32_t)n < 0 ? -1 : (int32_t)n;
}

/* *gpu: that of the call's tensors so far, -1 before the first; all are on the same one. */
static int same_gpu(int at, const char *what, int *gpu)
{
    if (*gpu < 0) *gpu = at;
    if (at == *gpu) return 0;
    PyErr_Format(PyExc_ValueError, "%s is on GPU %d and another tensor of the call on GPU %d", what, at, *gpu);
    return -1;
}

static int on_gpu(PyObject *t, const char *what, int *gpu)
{
    const int at = gpu_of(t);
    if (at == -2) return -1;
    return at < 0 ? refuse(PyExc_ValueError, what, "is not on a GPU") : same_gpu(at, what, gpu);
}

/* The library launches on the current GPU (the first one, before torch has looked for them). */
static int is_current(int gpu)
{
    uint64_t now = 0;
    if (gpu < 0) return 0;
    PyObject *known = PyObject_GetAttr(t_cuda, s_initialized);
    if (!known) return -1;
    const int ask = PyObject_IsTrue(known);
    Py_DECREF(known);
    if (ask < 0 || (ask && taken(PyObject_CallMethodNoArgs(t_c, s_get_current), as_size, &now))) return -1;
    if ((int32_t)now == gpu) return 0;
    PyErr_Format(PyExc_ValueError, "the tensors are on GPU %d and the current one is %d", gpu, (int)(int32_t)now);
    return -1;
}

/* A history that torch is recording would end here without a word. */
static int no_history(PyObject *t, const char *what)
{
    PyObject *v = PyObject_GetAttr(t, s_requires_grad);
    if (!v) return -1;
    const int wanted = PyObject_IsTrue(v);
    Py_DECREF(v);
    if (wanted <= 0) return wanted;
    v = PyObject_CallNoArgs(grad_enabled);
    if (!v) return -1;
    const int on = PyObject_IsTrue(v);
    Py_DECREF(v);
    return on <= 0 ? on
                   : refuse(PyExc_RuntimeError, what, "requires grad, and this call keeps no history: its gradients are calls of their own. Call it "
                                                      "in the forward of a torch.autograd.Function, under torch.no_grad(), or with detached tensors");
}

/* A 2-D tensor (deep: or a 3-D one, matrices one behind the other, *groups of them) as rows; ld as the library counts it. */
static int rows_of(PyObject *t, const char *what, int deep, int32_t *groups, int64_t *rows, int64_t *cols, int64_t *ld)
{
    int64_t n[3], by[3];
    const int dims = numbers(PyObject_GetAttr(t, s_shape), n);
    if (dims < 0) return -1;
    if (dims != 2 && !(deep && dims == 3)) return refuse(PyExc_ValueError, what, deep ? "is to be [groups, channels, columns]" : "is to be a matrix with contiguous rows");
    if (numbers(PyObject_CallMethodNoArgs(t, s_stride), by) < 0) return -1;
    if (dims == 2) {
        n[2] = n[1], by[2] = by[1], n[1] = n[0], by[1] = by[0];
        n[0] = 1, by[0] = 0;
    }
    if (n[2] > 1 && by[2] != 1 && n[0] > 0 && n[1] > 0) return refuse(PyExc_ValueError, what, "is to be a matrix with contiguous rows");
    if (n[0] > 1 && n[1] > 1 && by[0] != n[1] * by[1]) return refuse(PyExc_ValueError, what, "is to have its matrices one behind the other");
    *rows = n[0] * n[1];
    *cols = n[2];
    *ld = n[1] > 1 ? by[1] : n[0] > 1 ? by[0] : by[1] > n[2] ? by[1] : n[2];
    if (groups) *groups = (int32_t)n[0];
    return 0;
}

static int matrix(PyObject *t, const char *what, int deep, int32_t *groups, seer_dense *d, int *gpu)
{
    uint64_t at;
    if (rows_of(t, what, deep, groups, &d->rows, &d->cols, &d->ld) || on_gpu(t, what, gpu)) return -1;
    if ((d->type = type_of(t, what)) < 0 || (d->type <= SEER_F16 && no_history(t, what)) || address_of(t, &at)) return -1;
    d->data = (void *)(uintptr_t)at;
    return 0;
}

/* A contiguous tensor of n elements of a type; None: null. */
static int vector(PyObject *t, const char *what, int type, int64_t n, uint64_t *at, int *gpu)
{
    *at = 0;
    if (t == Py_None) return 0;
    uint64_t count;
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    const int same = d == types[type];
    Py_DECREF(d);
    const int whole = truth(t, s_is_contiguous), there = gpu_of(t);
    if (whole < 0 || there == -2 || taken(PyObject_CallMethodNoArgs(t, s_numel), as_size, &count)) return -1;
    if (!same || !whole || there < 0 || (int64_t)count != n) {
        PyErr_Format(PyExc_ValueError, "%s is to be a contiguous %S tensor of %lld elements on the GPU", what, types[type], (long long)n);
        return -1;
    }
    return same_gpu(there, what, gpu) || (type == SEER_F32 && no_history(t, what)) || address_of(t, at) ? -1 : 0;
}

/* An array of a routing. */
static int array_attr(PyObject *r, PyObject *name, const char *what, uint64_t *at, int *gpu)
{
    PyObject *t = PyObject_GetAttr(r, name);
    if (!t) return -1;
    const int rc = on_gpu(t, what, gpu) || address_of(t, at) ? -1 : 0;
    Py_DECREF(t);
    return rc;
}

/* all: with the order of the slots; else only choice_slot, which is all that rows go by. */
static int routing_of(PyObject *r, int all, seer_routing *c, int *gpu)
{
    uint64_t tokens, choices, experts, ptr = 0, order = 0, slots;
    if (size_attr(r, s_tokens, &tokens) || size_attr(r, s_choices, &choices) || size_attr(r, s_experts, &experts) ||
        array_attr(r, s_choice_slot, "choice_slot", &slots, gpu) ||
        (all && (array_attr(r, s_expert_ptr, "expert_ptr", &ptr, gpu) || array_attr(r, s_slot_choice, "slot_choice", &order, gpu))))
        return -1;
    c->tokens = (int32_t)tokens;
    c->choices = (int32_t)choices;
    c->experts = (int32_t)experts;
    c->expert_ptr = P(int32_t *, ptr);
    c->slot_choice = P(int32_t *, order);
    c->choice_slot = P(int32_t *, slots);
    return 0;
}

/* A contiguous tensor of any type, as bytes; None: null. */
static int space(PyObject *workspace, uint64_t *at, uint64_t *bytes, int *gpu)
{
    *at = *bytes = 0;
    if (workspace == Py_None) return 0;
    const int whole = truth(workspace, s_is_contiguous), there = gpu_of(workspace);
    if (whole < 0 || there == -2) return -1;
    if (!whole || there < 0) return refuse(PyExc_ValueError, "the workspace", "is to be contiguous and on the GPU");
    if (same_gpu(there, "the workspace", gpu)) return -1;
    return address_of(workspace, at) || taken(PyObject_GetAttr(workspace, s_nbytes), as_size, bytes) ? -1 : 0;
}

static int given(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return 0;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments", want);
    return -1;
}

#define ASYNC(call)                                                                                                                \
    int rc;                                                                                                                        \
    Py_BEGIN_ALLOW_THREADS                                                                                                         \
    rc = call;                                                                                                                     \
    Py_END_ALLOW_THREADS                                                                                                           \
    return PyLong_FromLong(rc)

static PyObject *m_route(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_routing r;
    uint64_t at, ws, bytes, stream;
    int gpu = -1;
    if (given(n, 4) || routing_of(a[1], 1, &r, &gpu)) return NULL;
    const int type = type_of(a[0], "expert");
    if (type < 0 || vector(a[0], "expert", type, (int64_t)r.tokens * r.choices, &at, &gpu) || space(a[2], &ws, &bytes, &gpu) ||
        as_size(a[3], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_route(P(const void *, at), type, &r, P(void *, ws), (size_t)bytes, P(void *, stream)));
}

/* (routing, matrix by token, matrix by slot, weight, stream), whichever way the rows go */
static int rows_parse(PyObject *const *a, Py_ssize_t n, const char *first, const char *second, seer_routing *r, seer_dense *x,
                      seer_dense *y, uint64_t *weight, uint64_t *stream)
{
    int gpu = -1;
    return given(n, 5) || routing_of(a[0], 0, r, &gpu) || matrix(a[1], first, 0, NULL, x, &gpu) || matrix(a[2], second, 0, NULL, y, &gpu) ||
           vector(a[3], "weight", SEER_F32, (int64_t)r->tokens * r->choices, weight, &gpu) || as_size(a[4], stream) || is_current(gpu);
}

static PyObject *m_gather(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_routing r;
    seer_dense x, out;
    uint64_t weight, stream;
    if (rows_parse(a, n, "x", "out", &r, &x, &out, &weight, &stream)) return NULL;
    ASYNC(f_gather(&r, &x, P(const float *, weight), &out, P(void *, stream)));
}

static PyObject *m_combine(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_routing r;
    seer_dense z, y;
    uint64_t weight, stream;
    if (rows_parse(a, n, "z", "y", &r, &z, &y, &weight, &stream)) return NULL;
    ASYNC(f_combine(&r, &z, P(const float *, weight), &y, P(void *, stream)));
}

/* (routing, dy, z or None, weight or None, dz or None, dweight or None, stream) */
static PyObject *m_grad(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_routing r;
    seer_dense dy, z, dz;
    uint64_t weight, dweight, stream;
    int gpu = -1;
    if (given(n, 7) || routing_of(a[0], 0, &r, &gpu) || matrix(a[1], "dy", 0, NULL, &dy, &gpu) ||
        (a[2] != Py_None && matrix(a[2], "z", 0, NULL, &z, &gpu)) ||
        vector(a[3], "weight", SEER_F32, (int64_t)r.tokens * r.choices, &weight, &gpu) ||
        (a[4] != Py_None && matrix(a[4], "dz", 0, NULL, &dz, &gpu)) ||
        vector(a[5], "dweight", SEER_F32, (int64_t)r.tokens * r.choices, &dweight, &gpu) || as_size(a[6], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_grad(&r, &dy, a[2] != Py_None ? &z : NULL, P(const float *, weight), a[4] != Py_None ? &dz : NULL, P(float *, dweight),
                 P(void *, stream)));
}

/* (routing or None, x, q, scale, stream) */
static PyObject *m_quantize(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_routing r;
    seer_dense x, q;
    uint64_t scale, stream;
    const int routed = n == 5 && a[0] != Py_None;
    int gpu = -1;
    if (given(n, 5) || (routed && routing_of(a[0], 0, &r, &gpu)) || matrix(a[1], "x", 0, NULL, &x, &gpu) || matrix(a[2], "q", 0, NULL, &q, &gpu) ||
        vector(a[3], "scale", SEER_F32, routed ? (int64_t)r.tokens * r.choices : x.rows, &scale, &gpu) || as_size(a[4], &stream) || is_current(gpu))
        return NULL;
    ASYNC(routed ? f_gather_i8(&r, &x, &q, P(float *, scale), P(void *, stream)) : f_quantize(&x, &q, P(float *, scale), P(void *, stream)));
}

/* (a, a_scale, b, b_scale, group_ptr or None, out, workspace or None, stream) */
static PyObject *m_product(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    seer_dense a, b, out;
    int32_t groups;
    uint64_t sa, sb, ptr, ws, bytes, stream;
    int gpu = -1;
    if (given(n, 8) || matrix(v[0], "a", 0, NULL, &a, &gpu) || vector(v[1], "a_scale", SEER_F32, a.rows, &sa, &gpu) ||
        matrix(v[2], "b", 1, &groups, &b, &gpu) || vector(v[3], "b_scale", SEER_F32, b.rows, &sb, &gpu) ||
        vector(v[4], "group_ptr", SEER_I32, (int64_t)groups + 1, &ptr, &gpu) || matrix(v[5], "out", 0, NULL, &out, &gpu) ||
        space(v[6], &ws, &bytes, &gpu) || as_size(v[7], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_product(&a, P(const float *, sa), &b, P(const float *, sb), P(const int32_t *, ptr), groups, &out, P(void *, ws), (size_t)bytes,
                    P(void *, stream)));
}

/* One tensor of a list of gradients. */
static int gradient(PyObject *t, uint64_t *at, uint64_t *n, int *type, int *gpu)
{
    const int there = gpu_of(t), whole = there == -2 ? -1 : truth(t, s_is_contiguous);
    if (whole < 0) return -1;
    if (there < 0 || !whole) return refuse(PyExc_ValueError, "gradients and outputs", "are to be contiguous and on the GPU");
    if (same_gpu(there, "a gradient or output", gpu)) return -1;
    if ((*type = type_of(t, "a gradient")) < 0) return -1;
    return address_of(t, at) || taken(PyObject_CallMethodNoArgs(t, s_numel), as_size, n) ? -1 : 0;
}

/* (list of gradients, list of outputs or None, address of the seer_grad array to fill, its length): the GPU that they are on, or -1 */
static PyObject *m_grads(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    uint64_t list, count;
    if (given(n, 4) || as_size(a[2], &list) || as_size(a[3], &count)) return NULL;
    const int apart = a[1] != Py_None;
    if (!PyList_Check(a[0]) || (apart && !PyList_Check(a[1]))) {
        PyErr_SetString(PyExc_TypeError, "lists are wanted");
        return NULL;
    }
    seer_grad *const out = P(seer_grad *, list);
    int gpu = -1;
    for (uint64_t i = 0; i < count; ++i) {
        if ((uint64_t)PyList_GET_SIZE(a[0]) != count || (apart && (uint64_t)PyList_GET_SIZE(a[1]) != count)) {
            PyErr_SetString(PyExc_ValueError, "as many outputs as gradients are wanted");
            return NULL;
        }
        uint64_t at, to, elems, room;
        int type, as;
        PyObject *g = PyList_GET_ITEM(a[0], (Py_ssize_t)i), *o = apart ? PyList_GET_ITEM(a[1], (Py_ssize_t)i) : g;
        Py_INCREF(g);
        Py_INCREF(o);
        int rc = gradient(g, &at, &elems, &type, &gpu);
        if (!rc && apart) rc = gradient(o, &to, &room, &as, &gpu);
        else to = at, room = elems, as = type;
        if (!rc && (as != type || room != elems)) rc = refuse(PyExc_ValueError, "an output", "is to have its gradient's type and size");
        if (!rc && type > SEER_F16) {
            PyErr_Format(PyExc_TypeError, "a gradient is %S", types[type]);
            rc = -1;
        }
        Py_DECREF(g);
        Py_DECREF(o);
        if (rc) return NULL;
        out[i].grad = P(const void *, at);
        out[i].out = P(void *, to);
        out[i].n = (int64_t)elems;
        out[i].type = type;
    }
    return PyLong_FromLong(gpu);
}

/* (address of the seer_grad array, count, max_norm or None, norm, workspace, stream, what m_grads returned) */
static PyObject *m_clip(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    uint64_t list, count, norm, ws, bytes, stream, tensors;
    if (given(n, 7) || as_size(a[0], &list) || as_size(a[1], &count) || as_size(a[5], &stream) || as_size(a[6], &tensors)) return NULL;
    int gpu = (int32_t)tensors;
    if (vector(a[3], "norm", SEER_F32, 1, &norm, &gpu) || space(a[4], &ws, &bytes, &gpu) || is_current(gpu)) return NULL;
    const int clip = a[2] != Py_None;
    const double most = clip ? PyFloat_AsDouble(a[2]) : 0;
    if (PyErr_Occurred()) return NULL;
    ASYNC(clip ? f_clip(P(const seer_grad *, list), (int32_t)count, (float)most, P(float *, norm), P(void *, ws), (size_t)bytes, P(void *, stream))
               : f_norm(P(const seer_grad *, list), (int32_t)count, P(float *, norm), P(void *, ws), (size_t)bytes, P(void *, stream)));
}

static PyObject *m_bind_routed(PyObject *self, PyObject *args)
{
    unsigned long long f[9];
    PyObject *t[6], *c, *cuda, *grad;
    if (!PyArg_ParseTuple(args, "KKKKKKKKKOOOOOOOOO", f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6, f + 7, f + 8, &c, &cuda, &grad, t, t + 1, t + 2,
                          t + 3, t + 4, t + 5))
        return NULL;
    f_route = P(int (*)(const void *, int32_t, const seer_routing *, void *, size_t, void *), f[0]);
    f_gather = P(int (*)(const seer_routing *, const seer_dense *, const float *, const seer_dense *, void *), f[1]);
    f_combine = P(int (*)(const seer_routing *, const seer_dense *, const float *, const seer_dense *, void *), f[2]);
    f_grad = P(int (*)(const seer_routing *, const seer_dense *, const seer_dense *, const float *, const seer_dense *, float *, void *), f[3]);
    f_quantize = P(int (*)(const seer_dense *, const seer_dense *, float *, void *), f[4]);
    f_gather_i8 = P(int (*)(const seer_routing *, const seer_dense *, const seer_dense *, float *, void *), f[5]);
    f_product = P(int (*)(const seer_dense *, const float *, const seer_dense *, const float *, const int32_t *, int32_t, const seer_dense *,
                          void *, size_t, void *), f[6]);
    f_norm = P(int (*)(const seer_grad *, int32_t, float *, void *, size_t, void *), f[7]);
    f_clip = P(int (*)(const seer_grad *, int32_t, float, float *, void *, size_t, void *), f[8]);
    Py_INCREF(grad);
    Py_XSETREF(grad_enabled, grad);
    Py_INCREF(c);
    Py_XSETREF(t_c, c);
    Py_INCREF(cuda);
    Py_XSETREF(t_cuda, cuda);
    for (int i = 0; i < 6; ++i) {
        Py_INCREF(t[i]);
        Py_XSETREF(types[i], t[i]);
    }
    Py_RETURN_NONE;
}

/* ---- what a routed layer is fed by: the router's choice (router.py) and the embedding of tokens (embedding.py) */

static int (*f_choose)(const seer_dense *, const float *, const seer_choice *, int32_t *, float *, void *);
static int (*f_choose_grad)(const seer_dense *, const seer_choice *, const int32_t *, const float *, const seer_dense *, void *);
static int (*f_embed)(const void *, int32_t, const seer_dense *, float, const seer_dense *, void *);
static int (*f_embed_grad)(const void *, int32_t, const seer_dense *, float, int32_t, const seer_dense *, void *, size_t, void *);

/* (logits, bias or None, address of the seer_choice, expert, weight, stream) */
static PyObject *m_choose(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_dense logits;
    uint64_t bias, how, expert, weight, stream;
    int gpu = -1;
    if (given(n, 6) || as_size(a[2], &how) || matrix(a[0], "logits", 0, NULL, &logits, &gpu)) return NULL;
    const int64_t count = logits.rows * P(const seer_choice *, how)->choices;
    if (vector(a[1], "bias", SEER_F32, logits.cols, &bias, &gpu) || vector(a[3], "expert", SEER_I32, count, &expert, &gpu) ||
        vector(a[4], "weight", SEER_F32, count, &weight, &gpu) || as_size(a[5], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_choose(&logits, P(const float *, bias), P(const seer_choice *, how), P(int32_t *, expert), P(float *, weight), P(void *, stream)));
}

/* (logits, address of the seer_choice, expert, dweight, dlogits, stream) */
static PyObject *m_choose_grad(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_dense logits, dlogits;
    uint64_t how, expert, dweight, stream;
    int gpu = -1;
    if (given(n, 6) || as_size(a[1], &how) || matrix(a[0], "logits", 0, NULL, &logits, &gpu)) return NULL;
    const int64_t count = logits.rows * P(const seer_choice *, how)->choices;
    if (vector(a[2], "expert", SEER_I32, count, &expert, &gpu) || vector(a[3], "dweight", SEER_F32, count, &dweight, &gpu) ||
        matrix(a[4], "dlogits", 0, NULL, &dlogits, &gpu) || as_size(a[5], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_choose_grad(&logits, P(const seer_choice *, how), P(const int32_t *, expert), P(const float *, dweight), &dlogits, P(void *, stream)));
}

static int number(PyObject *o, float *out)
{
    const double v = PyFloat_AsDouble(o);
    *out = (float)v;
    return v == -1.0 && PyErr_Occurred() ? -1 : 0;
}

/* Tokens, of a type that the library knows or refuses. */
static int tokens_of(PyObject *t, int64_t n, uint64_t *at, int *type, int *gpu)
{
    return (*type = type_of(t, "token")) < 0 || vector(t, "token", *type, n, at, gpu) ? -1 : 0;
}

/* (token, table, scale, out, stream) */
static PyObject *m_embed(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_dense table, out;
    uint64_t token, stream;
    float scale;
    int gpu = -1, type;
    if (given(n, 5) || matrix(a[1], "table", 0, NULL, &table, &gpu) || number(a[2], &scale) || matrix(a[3], "out", 0, NULL, &out, &gpu) ||
        tokens_of(a[0], out.rows, &token, &type, &gpu) || as_size(a[4], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_embed(P(const void *, token), type, &table, scale, &out, P(void *, stream)));
}

/* (token, dy, scale, accumulate, dtable, workspace or None, stream) */
static PyObject *m_embed_grad(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_dense dy, dtable;
    uint64_t token, ws, bytes, stream;
    float scale;
    int gpu = -1, type;
    if (given(n, 7) || matrix(a[1], "dy", 0, NULL, &dy, &gpu) || number(a[2], &scale) || matrix(a[4], "dtable", 0, NULL, &dtable, &gpu) ||
        tokens_of(a[0], dy.rows, &token, &type, &gpu) || space(a[5], &ws, &bytes, &gpu) || as_size(a[6], &stream) || is_current(gpu))
        return NULL;
    const int add = PyObject_IsTrue(a[3]);
    if (add < 0) return NULL;
    ASYNC(f_embed_grad(P(const void *, token), type, &dy, scale, add, &dtable, P(void *, ws), (size_t)bytes, P(void *, stream)));
}

static PyObject *m_bind_tokens(PyObject *self, PyObject *args)
{
    unsigned long long f[4];
    if (!PyArg_ParseTuple(args, "KKKK", f, f + 1, f + 2, f + 3)) return NULL;
    f_choose = P(int (*)(const seer_dense *, const float *, const seer_choice *, int32_t *, float *, void *), f[0]);
    f_choose_grad = P(int (*)(const seer_dense *, const seer_choice *, const int32_t *, const float *, const seer_dense *, void *), f[1]);
    f_embed = P(int (*)(const void *, int32_t, const seer_dense *, float, const seer_dense *, void *), f[2]);
    f_embed_grad = P(int (*)(const void *, int32_t, const seer_dense *, float, int32_t, const seer_dense *, void *, size_t, void *), f[3]);
    Py_RETURN_NONE;
}

/* ---- rows in 4-bit floating point (mx4.py) */

static int (*f_mx4_quantize)(const seer_dense *, const seer_mx4 *, void *);
static int (*f_gather_mx4)(const seer_routing *, const seer_dense *, const seer_mx4 *, void *);
static int (*f_mx4_product)(const seer_mx4 *, const seer_mx4 *, const int32_t *, int32_t, const seer_dense *, void *, size_t, void *);
static PyObject *type_u8;

static int bytes_of(PyObject *t, const char *what, int deep, int32_t *groups, int64_t *rows, int64_t *cols, int64_t *ld, void **data, int *gpu)
{
    uint64_t at;
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    Py_DECREF(d);                            /* (torch keeps its types) */
    if (d != type_u8) return refuse(PyExc_TypeError, what, "is to be a uint8 tensor");
    if (rows_of(t, what, deep, groups, rows, cols, ld) || on_gpu(t, what, gpu) || address_of(t, &at)) return -1;
    *data = (void *)(uintptr_t)at;
    return 0;
}

/* Codes, 16 bytes to a block, and a scale byte for each; all blocks count as whole. */
static int blocks_of(PyObject *q, const char *q_what, PyObject *scale, const char *scale_what, int deep, int32_t *groups, seer_mx4 *m, int *gpu)
{
    int32_t scale_groups;
    int64_t rows, bytes, blocks;
    if (bytes_of(q, q_what, deep, groups, &m->rows, &bytes, &m->ld, &m->data, gpu) ||
        bytes_of(scale, scale_what, deep, &scale_groups, &rows, &blocks, &m->scale_ld, &m->scale, gpu))
        return -1;
    if (rows != m->rows || bytes != 16 * blocks || (groups && scale_groups != *groups))
        return refuse(PyExc_ValueError, scale_what, "is to have a byte for every 16 bytes of the codes");
    m->cols = 32 * blocks;
    return 0;
}

/* (routing or None, x, q, scale, stream) */
static PyObject *m_mx4_quantize(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    seer_routing r;
    seer_dense x;
    seer_mx4 q;
    uint64_t stream;
    const int routed = n == 5 && a[0] != Py_None;
    int gpu = -1;
    if (given(n, 5) || (routed && routing_of(a[0], 0, &r, &gpu)) || matrix(a[1], "x", 0, NULL, &x, &gpu) ||
        blocks_of(a[2], "q", a[3], "scale", 0, NULL, &q, &gpu) || as_size(a[4], &stream) || is_current(gpu))
        return NULL;
    if (q.cols / 32 != (x.cols + 31) / 32) {
        refuse(PyExc_ValueError, "q", "is to have 16 bytes for every 32 columns of x");
        return NULL;
    }
    q.cols = x.cols;
    ASYNC(routed ? f_gather_mx4(&r, &x, &q, P(void *, stream)) : f_mx4_quantize(&x, &q, P(void *, stream)));
}

/* (a, a_scale, b, b_scale, group_ptr or None, out, workspace or None, stream) */
static PyObject *m_mx4_product(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    seer_mx4 a, b;
    seer_dense out;
    int32_t groups;
    uint64_t ptr, ws, bytes, stream;
    int gpu = -1;
    if (given(n, 8) || blocks_of(v[0], "a", v[1], "a_scale", 0, NULL, &a, &gpu) || blocks_of(v[2], "b", v[3], "b_scale", 1, &groups, &b, &gpu) ||
        vector(v[4], "group_ptr", SEER_I32, (int64_t)groups + 1, &ptr, &gpu) || matrix(v[5], "out", 0, NULL, &out, &gpu) ||
        space(v[6], &ws, &bytes, &gpu) || as_size(v[7], &stream) || is_current(gpu))
        return NULL;
    ASYNC(f_mx4_product(&a, &b, P(const int32_t *, ptr), groups, &out, P(void *, ws), (size_t)bytes, P(void *, stream)));
}

static PyObject *m_bind_mx4(PyObject *self, PyObject *args)
{
    unsigned long long f[3];
    PyObject *u8;
    if (!PyArg_ParseTuple(args, "KKKO", f, f + 1, f + 2, &u8)) return NULL;
    f_mx4_quantize = P(int (*)(const seer_dense *, const seer_mx4 *, void *), f[0]);
    f_gather_mx4 = P(int (*)(const seer_routing *, const seer_dense *, const seer_mx4 *, void *), f[1]);
    f_mx4_product = P(int (*)(const seer_mx4 *, const seer_mx4 *, const int32_t *, int32_t, const seer_dense *, void *, size_t, void *), f[2]);
    Py_INCREF(u8);
    Py_XSETREF(type_u8, u8);
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", m_bind, METH_VARARGS, "bind(spmv, spmv_auto, spmv_model, spmv_prepared): addresses of the library's functions"},
    {"spmv", (PyCFunction)(void (*)(void))m_spmv, METH_FASTCALL, "spmv(kernel_id, A, x, y, workspace, stream) -> status"},
    {"spmv_auto", (PyCFunction)(void (*)(void))m_auto, METH_FASTCALL, "spmv_auto(tree address, A, x, y, workspace, stream) -> status"},
    {"spmv_model", (PyCFunction)(void (*)(void))m_model, METH_FASTCALL,
     "spmv_model(model address, A, x, y, workspace, stream) -> (status, path, kernel id)"},
    {"spmv_prepared", (PyCFunction)(void (*)(void))m_prepared, METH_FASTCALL,
     "spmv_prepared(plan address, A, x, y, workspace, stream) -> status"},
    {"bind_routed", m_bind_routed, METH_VARARGS, "bind_routed(addresses of the routed layer's functions, torch._C, torch.cuda, whether a history is recorded, torch's dtypes)"},
    {"route", (PyCFunction)(void (*)(void))m_route, METH_FASTCALL, "route(expert, routing, workspace, stream) -> status"},
    {"gather", (PyCFunction)(void (*)(void))m_gather, METH_FASTCALL, "gather(routing, x, out, weight, stream) -> status"},
    {"combine", (PyCFunction)(void (*)(void))m_combine, METH_FASTCALL, "combine(routing, z, y, weight, stream) -> status"},
    {"grad", (PyCFunction)(void (*)(void))m_grad, METH_FASTCALL, "grad(routing, dy, z, weight, dz, dweight, stream) -> status"},
    {"quantize", (PyCFunction)(void (*)(void))m_quantize, METH_FASTCALL, "quantize(routing, x, q, scale, stream) -> status"},
    {"product", (PyCFunction)(void (*)(void))m_product, METH_FASTCALL,
     "product(a, a_scale, b, b_scale, group_ptr, out, workspace, stream) -> status"},
    {"grads", (PyCFunction)(void (*)(void))m_grads, METH_FASTCALL, "grads(gradients, outputs or None, list address, count) -> GPU"},
    {"clip", (PyCFunction)(void (*)(void))m_clip, METH_FASTCALL, "clip(list address, count, max_norm, norm, workspace, stream, GPU) -> status"},
    {"bind_tokens", m_bind_tokens, METH_VARARGS, "bind_tokens(addresses of seer_route_choose, seer_route_choose_grad, seer_embed, seer_embed_grad)"},
    {"choose", (PyCFunction)(void (*)(void))m_choose, METH_FASTCALL, "choose(logits, bias or None, choice address, expert, weight, stream) -> status"},
    {"choose_grad", (PyCFunction)(void (*)(void))m_choose_grad, METH_FASTCALL,
     "choose_grad(logits, choice address, expert, dweight, dlogits, stream) -> status"},
    {"embed", (PyCFunction)(void (*)(void))m_embed, METH_FASTCALL, "embed(token, table, scale, out, stream) -> status"},
    {"embed_grad", (PyCFunction)(void (*)(void))m_embed_grad, METH_FASTCALL,
     "embed_grad(token, dy, scale, accumulate, dtable, workspace, stream) -> status"},
    {"bind_mx4", m_bind_mx4, METH_VARARGS, "bind_mx4(addresses of seer_mx4_quantize, seer_route_gather_mx4, seer_mx4_product, torch.uint8)"},
    {"mx4_quantize", (PyCFunction)(void (*)(void))m_mx4_quantize, METH_FASTCALL, "mx4_quantize(routing or None, x, q, scale, stream) -> status"},
    {"mx4_product", (PyCFunction)(void (*)(void))m_mx4_product, METH_FASTCALL,
     "mx4_product(a, a_scale, b, b_scale, group_ptr, out, workspace, stream) -> status"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of the asynchronous calls", -1,
                                    methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void)
{
    s_rows = PyUnicode_InternFromString("rows");
    s_cols = PyUnicode_InternFromString("cols");
    s_nnz = PyUnicode_InternFromString("nnz");
    s_row_ptr = PyUnicode_InternFromString("row_ptr");
    s_col_idx = PyUnicode_InternFromString("col_idx");
    s_values = PyUnicode_InternFromString("values");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    PyObject **const names[] = {&s_shape, &s_stride, &s_dtype, &s_get_device, &s_initialized, &s_get_current, &s_requires_grad, &s_is_contiguous, &s_tokens, &s_choices, &s_experts, &s_expert_ptr,
                                &s_slot_choice, &s_choice_slot, &s_nbytes};
    const char *const spelt[] = {"shape", "stride", "dtype", "get_device", "_initialized", "_cuda_getDevice", "requires_grad", "is_contiguous", "tokens", "choices", "experts", "expert_ptr",
                                 "slot_choice", "choice_slot", "nbytes"};
    for (size_t i = 0; i < sizeof spelt / sizeof *spelt; ++i)
        if (!(*names[i] = PyUnicode_InternFromString(spelt[i]))) return NULL;
    if (!s_rows || !s_cols || !s_nnz || !s_row_ptr || !s_col_idx || !s_values || !s_data_ptr || !s_numel) return NULL;
    return PyModule_Create(&module);
}
