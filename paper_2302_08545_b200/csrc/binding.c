/*
 * Argument marshalling of thc.Context in C: tensors -> device addresses, then the C ABI of
 * include/thc.h.  A round is four calls with up to 2 n + 4 addresses each; collected in Python
 * (a ctypes array per pointer list) that took longer than the kernels of a small round.
 *
 * Every function takes the context handle as an integer (0 where the call has none) and returns
 * the library's return code.  A tensor argument is anything with data_ptr(), a raw address as int,
 * or None (NULL).  A stream is None (the current stream of the current device), a raw handle as
 * int, or anything with cuda_stream.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "../../include/thc.h"

static PyObject *s_data_ptr, *s_nbytes, *s_cuda_stream;   /* interned names */
static PyObject *get_device, *get_raw_stream;             /* torch._C, looked up on first use */

/* Address of one argument; -1 with an exception set on failure. */
static int address(PyObject *o, void **p)
{
    if (o == Py_None) { *p = NULL; return 0; }
    if (PyLong_Check(o)) {
        *p = PyLong_AsVoidPtr(o);
        return PyErr_Occurred() ? -1 : 0;
    }
    PyObject *v = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (v == NULL) return -1;
    *p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

/* A list of addresses.  Longer lists than the library serves (THC_MAX_WORKERS) keep their length,
 * which the library refuses before it reads the array. */
typedef struct { void *p[THC_MAX_WORKERS]; uint32_t n; int given; } list_t;

static int addresses(PyObject *o, list_t *out)
{
    out->n = 0;
    out->given = o != Py_None;
    if (!out->given) return 0;
    PyObject *seq = PySequence_Fast(o, "a sequence of tensors is expected");
    if (seq == NULL) return -1;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    int rc = 0;
    for (Py_ssize_t i = 0; rc == 0 && i < n && i < (Py_ssize_t)THC_MAX_WORKERS; ++i)
        rc = address(PySequence_Fast_GET_ITEM(seq, i), &out->p[i]);
    out->n = (uint32_t)n;
    Py_DECREF(seq);
    return rc;
}

static void **array_of(list_t *l) { return l->given ? l->p : NULL; }

/* Another list (packed, rotated, ...) has to have an entry for each of the first one's n. */
static int same_length(const list_t *a, const list_t *b)
{
    if (!b->given || b->n >= a->n) return 0;
    PyErr_SetString(PyExc_ValueError, "the lists of per-worker tensors differ in length");
    return -1;
}

static int number(PyObject *o, uint64_t *v)
{
    *v = PyLong_AsUnsignedLongLong(o);
    return *v == (uint64_t)-1 && PyErr_Occurred() ? -1 : 0;
}

static int number32(PyObject *o, uint32_t *v)
{
    const unsigned long long x = PyLong_AsUnsignedLongLongMask(o);
    if (x == (unsigned long long)-1 && PyErr_Occurred()) return -1;
    *v = (uint32_t)x;
    return 0;
}

/* Workspace: its address and its size in bytes (None: no workspace). */
static int workspace(PyObject *o, void **p, uint64_t *bytes)
{
    *bytes = 0;
    if (address(o, p) != 0) return -1;
    if (o == Py_None) return 0;
    PyObject *v = PyObject_GetAttr(o, s_nbytes);
    if (v == NULL) return -1;
    const int rc = number(v, bytes);
    Py_DECREF(v);
    return rc;
}

static int stream_of(PyObject *o, void **st)
{
    PyObject *v;
    if (PyLong_Check(o)) {
        *st = PyLong_AsVoidPtr(o);
        return PyErr_Occurred() ? -1 : 0;
    }
    if (o == Py_None) {
        if (get_raw_stream == NULL) {
            PyObject *c = PyImport_ImportModule("torch._C");
            if (c == NULL) return -1;
            get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
            get_raw_stream = get_device ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : NULL;
            Py_DECREF(c);
            if (get_raw_stream == NULL) return -1;
        }
        PyObject *dev = PyObject_CallNoArgs(get_device);
        if (dev == NULL) return -1;
        v = PyObject_CallOneArg(get_raw_stream, dev);
        Py_DECREF(dev);
    } else {
        v = PyObject_GetAttr(o, s_cuda_stream);
    }
    if (v == NULL) return -1;
    *st = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

static int want(Py_ssize_t got, Py_ssize_t n)
{
    if (got == n) return 0;
    PyErr_Format(PyExc_TypeError, "%zd arguments are expected, got %zd", n, got);
    return -1;
}

#define ARGS PyObject *self, PyObject *const *a, Py_ssize_t na
#define BEGIN(count)                                                            \
    void *ctx_p, *st;                                                           \
    (void)self;                                                                 \
    if (want(na, count) || address(a[0], &ctx_p) || stream_of(a[na - 1], &st)) return NULL; \
    thc_ctx *ctx = (thc_ctx *)ctx_p;                                            \
    (void)ctx;                                                                  \
    int rc
#define CALL(expr)                                                              \
    Py_BEGIN_ALLOW_THREADS                                                      \
    rc = (expr);                                                                \
    Py_END_ALLOW_THREADS                                                        \
    return PyLong_FromLong(rc)

typedef const void *const *in_t;
typedef float *const *rot_t;

/* (handle, grads, d, scales, workspace, stream) */
static PyObject *b_prepare(ARGS)
{
    BEGIN(6);
    list_t g;
    uint64_t d, wb;
    void *scales, *ws;
    if (addresses(a[1], &g) || number(a[2], &d) || address(a[3], &scales) || workspace(a[4], &ws, &wb)) return NULL;
    CALL(thc_prepare(ctx, (in_t)g.p, g.n, d, scales, ws, wb, st));
}

/* (handle, grads, d, round, scales, rotated, workspace, stream) */
static PyObject *b_prepare_minmax(ARGS)
{
    BEGIN(8);
    list_t g, r;
    uint64_t d, wb;
    uint32_t rnd;
    void *scales, *ws;
    if (addresses(a[1], &g) || number(a[2], &d) || number32(a[3], &rnd) || address(a[4], &scales) ||
        addresses(a[5], &r) || same_length(&g, &r) || workspace(a[6], &ws, &wb)) return NULL;
    CALL(thc_prepare_minmax(ctx, (in_t)g.p, g.n, d, rnd, scales, (rot_t)array_of(&r), ws, wb, st));
}

/* (handle, grads, worker_base, d, round, scales, packed, rotated, workspace, stream) */
static PyObject *compress(ARGS, int with_scales)
{
    BEGIN(10);
    list_t g, p, r;
    uint64_t d, wb;
    uint32_t base, rnd;
    void *scales, *ws;
    if (addresses(a[1], &g) || number32(a[2], &base) || number(a[3], &d) || number32(a[4], &rnd) ||
        address(a[5], &scales) || addresses(a[6], &p) || addresses(a[7], &r) || same_length(&g, &p) ||
        same_length(&g, &r) || workspace(a[8], &ws, &wb)) return NULL;
    CALL(with_scales ? thc_prepare_compress(ctx, (in_t)g.p, g.n, base, d, rnd, scales, p.p, (rot_t)array_of(&r), ws, wb, st)
                     : thc_compress(ctx, (in_t)g.p, g.n, base, d, rnd, scales, p.p, (rot_t)array_of(&r), ws, wb, st));
}
static PyObject *b_compress(ARGS) { return compress(self, a, na, 0); }
static PyObject *b_prepare_compress(ARGS) { return compress(self, a, na, 1); }

/* (handle, rotated, worker_base, d, round, scales, packed, stream) */
static PyObject *b_quantize_rotated(ARGS)
{
    BEGIN(8);
    list_t r, p;
    uint64_t d;
    uint32_t base, rnd;
    void *scales;
    if (addresses(a[1], &r) || number32(a[2], &base) || number(a[3], &d) || number32(a[4], &rnd) ||
        address(a[5], &scales) || addresses(a[6], &p) || same_length(&r, &p)) return NULL;
    CALL(thc_quantize_rotated(ctx, (const float *const *)r.p, r.n, base, d, rnd, scales, p.p, st));
}

/* (handle, packed, d, total, stream) */
static PyObject *b_aggregate(ARGS)
{
    BEGIN(5);
    list_t p;
    uint64_t d;
    void *total;
    if (addresses(a[1], &p) || number(a[2], &d) || address(a[3], &total)) return NULL;
    CALL(thc_aggregate(ctx, (in_t)p.p, p.n, d, total, st));
}

/* (handle, total, divisor, d, round, scales, out, workspace, stream) */
static PyObject *b_decompress(ARGS)
{
    BEGIN(9);
    uint64_t d, wb;
    uint32_t divisor, rnd;
    void *total, *scales, *out, *ws;
    if (address(a[1], &total) || number32(a[2], &divisor) || number(a[3], &d) || number32(a[4], &rnd) ||
        address(a[5], &scales) || address(a[6], &out) || workspace(a[7], &ws, &wb)) return NULL;
    CALL(thc_decompress(ctx, total, divisor, d, rnd, scales, out, ws, wb, st));
}

/* (handle, packed, d, round, scales, out, total, workspace, stream) */
static PyObject *b_aggregate_decompress(ARGS)
{
    BEGIN(9);
    list_t p;
    uint64_t d, wb;
    uint32_t rnd;
    void *scales, *out, *total, *ws;
    if (addresses(a[1], &p) || number(a[2], &d) || number32(a[3], &rnd) || address(a[4], &scales) ||
        address(a[5], &out) || address(a[6], &total) || workspace(a[7], &ws, &wb)) return NULL;
    CALL(thc_aggregate_decompress(ctx, (in_t)p.p, p.n, d, rnd, scales, out, total, ws, wb, st));
}

/* (handle, grads, packed, d, round, scales, ef, workspace, stream) */
static PyObject *b_error_feedback(ARGS)
{
    BEGIN(9);
    list_t g, p, e;
    uint64_t d, wb;
    uint32_t rnd;
    void *scales, *ws;
    if (addresses(a[1], &g) || addresses(a[2], &p) || number(a[3], &d) || number32(a[4], &rnd) ||
        address(a[5], &scales) || addresses(a[6], &e) || same_length(&g, &p) || same_length(&g, &e) ||
        workspace(a[7], &ws, &wb)) return NULL;
    CALL(thc_error_feedback(ctx, (in_t)g.p, (in_t)p.p, g.n, d, rnd, scales, (rot_t)e.p, ws, wb, st));
}

/* (handle, grads, ef, d, stream) */
static PyObject *b_accumulate_error(ARGS)
{
    BEGIN(5);
    list_t g, e;
    uint64_t d;
    if (addresses(a[1], &g) || addresses(a[2], &e) || same_length(&g, &e) || number(a[3], &d)) return NULL;
    CALL(thc_accumulate_error(ctx, (rot_t)g.p, (const float *const *)e.p, g.n, d, st));
}

/* (0, grads, d, log2_block, in_dtype, t_p, scales, status, stream) */
static PyObject *b_prepare_noalloc(ARGS)
{
    BEGIN(9);
    list_t g;
    uint64_t d;
    uint32_t k, dtype;
    void *scales, *status;
    const double t_p = na > 5 ? PyFloat_AsDouble(a[5]) : 0.0;
    if (PyErr_Occurred()) return NULL;
    if (addresses(a[1], &g) || number(a[2], &d) || number32(a[3], &k) || number32(a[4], &dtype) ||
        address(a[6], &scales) || address(a[7], &status)) return NULL;
    CALL(thc_prepare_noalloc((in_t)g.p, g.n, d, k, dtype, t_p, scales, status, st));
}

/* ---- lists of tensors.  What these calls take besides is as long as the list says; a torch tensor that is
 * shorter, of another type, not contiguous or elsewhere is refused here, as the library sees only its address.
 *
 * A call looks at up to nine tensors, five attributes each: asked for one by one through Python that takes 0.4 us a
 * tensor, more than the launches of a small call.  torch describes a tensor in one C call through the exchange
 * table of the DLPack standard (version 1.3: type and layout of the structures below are the standard's); where
 * that is missing or does not want to, the attributes are asked for. */
typedef struct { int32_t type, id; } dl_device;
typedef struct { uint8_t code, bits; uint16_t lanes; } dl_type;
typedef struct { void *data; dl_device device; int32_t ndim; dl_type dtype; int64_t *shape, *strides; uint64_t byte_offset; } dl_tensor;
typedef struct {
    uint32_t major, minor;
    void *previous;
    void *allocate, *managed_from_object, *managed_to_object;
    int (*describe)(void *object, dl_tensor *out);
    int (*current_stream)(int32_t device_type, int32_t device, void **out);
} dl_exchange;
enum { DL_CPU = 1, DL_CUDA = 2, DL_INT = 0, DL_FLOAT = 2, DL_BFLOAT = 4 };

static PyObject *s_dtype, *s_is_contiguous, *s_get_device;
static PyObject *tensor_type, *t_f32, *t_bf16, *t_i64;    /* of torch, looked up on first use */
static const dl_exchange *exchange;                       /* null: attributes */

static int torch_names(void)
{
    if (t_i64 != NULL) return 0;
    PyObject *m = PyImport_ImportModule("torch");
    if (m == NULL) return -1;
    if (tensor_type == NULL) tensor_type = PyObject_GetAttrString(m, "Tensor");
    if (t_f32 == NULL) t_f32 = PyObject_GetAttrString(m, "float32");
    if (t_bf16 == NULL) t_bf16 = PyObject_GetAttrString(m, "bfloat16");
    if (tensor_type != NULL && t_f32 != NULL && t_bf16 != NULL) {
        PyObject *c = PyObject_GetAttrString(tensor_type, "__dlpack_c_exchange_api__");
        if (c != NULL) exchange = PyCapsule_GetPointer(c, "dlpack_exchange_api");
        Py_XDECREF(c);                                    /* (the table is static) */
        PyErr_Clear();
        if (exchange != NULL && (exchange->major != 1 || exchange->describe == NULL)) exchange = NULL;
        t_i64 = PyObject_GetAttrString(m, "int64");
    }
    Py_DECREF(m);
    return t_i64 != NULL ? 0 : -1;
}

static int list_of(PyObject *o, thc_tensors **list, thc_tensors_sizes_t *sz)
{
    void *p;
    memset(sz, 0, sizeof *sz);
    if (address(o, &p) != 0 || torch_names() != 0) return -1;
    *list = (thc_tensors *)p;
    if (p != NULL) thc_tensors_sizes(*list, sz);
    return 0;
}

/* The stream of a call on a list: None is the current one of the list's device. */
static int list_stream(PyObject *o, const thc_tensors_sizes_t *sz, void **st)
{
    if (o == Py_None && exchange != NULL && exchange->current_stream != NULL && sz->n != 0 && sz->device >= 0) {
        if (exchange->current_stream(DL_CUDA, sz->device, st) == 0) return 0;
        PyErr_Clear();
    }
    return stream_of(o, st);
}

/* What a tensor is, if it is contiguous and on the list's device (1; else 0, or -1 with an exception set).  `type` is NULL where torch's
 * table describes it, which then tells in `kind`. */
typedef struct { void *p; uint64_t bytes; PyObject *type; dl_type kind; } block_t;
static int block_of(PyObject *o, const thc_tensors_sizes_t *sz, block_t *b)
{
    dl_tensor d;
    memset(&d, 0, sizeof d);
    memset(b, 0, sizeof *b);
    if (exchange != NULL && exchange->describe(o, &d) == 0) {
        uint64_t n = 1;
        int ok = 1;
        for (int32_t i = d.ndim; i-- > 0;) {
            if (d.strides != NULL && d.shape[i] > 1 && d.strides[i] != (int64_t)n) ok = 0;
            n *= (uint64_t)d.shape[i];
        }
        const int cuda = d.device.type == DL_CUDA;
        b->p = (char *)d.data + d.byte_offset;
        b->bytes = n * d.dtype.bits / 8u * d.dtype.lanes;
        b->kind = d.dtype;
        return ok && (cuda || d.device.type == DL_CPU) && (cuda ? d.device.id : -1) == sz->device;
    }
    PyErr_Clear();
    if (address(o, &b->p) != 0) return -1;
    PyObject *t = PyObject_GetAttr(o, s_dtype), *c = PyObject_CallMethodNoArgs(o, s_is_contiguous), *v = PyObject_GetAttr(o, s_nbytes),
             *g = PyObject_CallMethodNoArgs(o, s_get_device);
    int ok = t != NULL && c != NULL && v != NULL && g != NULL && number(v, &b->bytes) == 0;
    const long device = ok ? PyLong_AsLong(g) : 0;
    ok = ok && c == Py_True && device == sz->device;
    b->type = t;                                          /* (torch's types are never freed) */
    Py_XDECREF(t);
    Py_XDECREF(c);
    Py_XDECREF(v);
    Py_XDECREF(g);
    return PyErr_Occurred() ? -1 : ok;
}

enum { F32, BF16, I64 };
static int vector(PyObject *o, void **p, int type, uint64_t elements, const thc_tensors_sizes_t *sz, const char *what)
{
    if (o == Py_None || PyLong_Check(o) || sz->n == 0) return address(o, p);
    const int is = PyObject_IsInstance(o, tensor_type);
    if (is < 0) return -1;
    if (is == 0) return address(o, p);
    block_t b;
    int ok = block_of(o, sz, &b);
    if (ok < 0) return -1;
    const uint32_t size = type == F32 ? 4u : type == BF16 ? 2u : 8u;
    if (b.type != NULL) ok = ok && b.type == (type == F32 ? t_f32 : type == BF16 ? t_bf16 : t_i64);
    else ok = ok && b.kind.lanes == 1 && b.kind.bits == size * 8u && b.kind.code == (type == F32 ? DL_FLOAT : type == BF16 ? DL_BFLOAT : DL_INT);
    *p = b.p;
    if (ok && b.bytes >= elements * size) return 0;
    PyErr_Format(PyExc_ValueError, "%s: a contiguous %s tensor of at least %llu elements on the context's device is expected", what,
                 type == F32 ? "float32" : type == BF16 ? "bfloat16" : "int64", (unsigned long long)elements);
    return -1;
}

/* Workspace of a call on a list: a tensor of any type, contiguous and on the list's device; anything else as for the other calls. */
static int list_workspace(PyObject *o, void **p, uint64_t *bytes, const thc_tensors_sizes_t *sz)
{
    if (o == Py_None || sz->n == 0) return workspace(o, p, bytes);
    const int is = PyObject_IsInstance(o, tensor_type);
    if (is < 0) return -1;
    if (is == 0) return workspace(o, p, bytes);
    block_t b;
    const int ok = block_of(o, sz, &b);
    if (ok < 0) return -1;
    *p = b.p;
    *bytes = b.bytes;
    if (ok && b.p != NULL) return 0;
    PyErr_SetString(PyExc_ValueError, "workspace: a contiguous tensor on the context's device is expected");
    return -1;
}

/* One vector per worker. */
static int vectors(PyObject *o, list_t *out, int type, const thc_tensors_sizes_t *sz, const char *what)
{
    out->n = 0;
    out->given = o != Py_None;
    if (!out->given) return 0;
    PyObject *seq = PySequence_Fast(o, "a sequence of tensors is expected");
    if (seq == NULL) return -1;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    int rc = 0;
    if (sz->n != 0 && n != (Py_ssize_t)sz->n) {
        PyErr_Format(PyExc_ValueError, "%s: one per worker is expected", what);
        rc = -1;
    }
    for (Py_ssize_t i = 0; rc == 0 && i < n && i < (Py_ssize_t)THC_MAX_WORKERS; ++i)
        rc = vector(PySequence_Fast_GET_ITEM(seq, i), &out->p[i], type, sz->d, sz, what);
    out->n = (uint32_t)n;
    Py_DECREF(seq);
    return rc;
}

static int real(PyObject *o, double *v)
{
    *v = PyFloat_AsDouble(o);
    return *v == -1.0 && PyErr_Occurred() ? -1 : 0;
}

/* `at`: the list's place among the arguments */
#define LIST_CALL(count, at)                                                    \
    void *ctx_p, *st, *ws;                                                      \
    thc_tensors *list;                                                          \
    thc_tensors_sizes_t sz;                                                     \
    uint64_t wb;                                                                \
    int rc;                                                                     \
    (void)self;                                                                 \
    if (want(na, count) || address(a[0], &ctx_p) || list_of(a[at], &list, &sz) || list_stream(a[na - 1], &sz, &st)) return NULL; \
    thc_ctx *ctx = (thc_ctx *)ctx_p

/* (handle, list, norms, workspace, stream) */
static PyObject *b_grad_norm(ARGS)
{
    LIST_CALL(5, 1);
    void *norms;
    if (vector(a[2], &norms, F32, sz.n, &sz, "norms") || list_workspace(a[3], &ws, &wb, &sz)) return NULL;
    CALL(thc_grad_norm(ctx, list, norms, ws, wb, st));
}

/* (handle, list, max_norm, out, norms, workspace, stream) */
static PyObject *b_clip_grads(ARGS)
{
    LIST_CALL(7, 1);
    double most;
    void *out, *norms;
    if (real(a[2], &most) || address(a[3], &out) || vector(a[4], &norms, F32, sz.n, &sz, "norms") ||
        list_workspace(a[5], &ws, &wb, &sz)) return NULL;
    CALL(thc_clip_grads(ctx, list, most, out, norms, ws, wb, st));
}

/* (handle, list, max_norm, ef, flats, norms, workspace, bf16, stream) */
static PyObject *b_gather_grads(ARGS)
{
    LIST_CALL(9, 1);
    double most;
    list_t e, f;
    void *norms;
    const int type = PyObject_IsTrue(a[7]) ? BF16 : F32;
    if (real(a[2], &most) || vectors(a[3], &e, F32, &sz, "ef") || vectors(a[4], &f, type, &sz, "flats") ||
        vector(a[5], &norms, F32, sz.n, &sz, "norms") || list_workspace(a[6], &ws, &wb, &sz)) return NULL;
    CALL(thc_gather_grads(ctx, list, most, (const float *const *)array_of(&e), array_of(&f), norms, ws, wb, st));
}

/* (handle, list, max_norm, norms, scales, out, grads, ef, stream) */
static PyObject *b_void_round(ARGS)
{
    void *ctx_p, *st, *norms, *scales, *out;
    thc_tensors *list;
    thc_tensors_sizes_t sz;
    thc_sizes_t round;
    list_t g, e;
    double most;
    int rc;
    (void)self;
    if (want(na, 9) || address(a[0], &ctx_p) || list_of(a[1], &list, &sz) || list_stream(a[8], &sz, &st) || real(a[2], &most)) return NULL;
    memset(&round, 0, sizeof round);
    if (ctx_p != NULL && sz.n != 0) thc_sizes(ctx_p, sz.d, 1, &round);
    if (vector(a[3], &norms, F32, sz.n, &sz, "norms") || vector(a[4], &scales, F32, round.scales_count, &sz, "scales") ||
        vector(a[5], &out, F32, sz.d, &sz, "out") || vectors(a[6], &g, F32, &sz, "grads") || vectors(a[7], &e, F32, &sz, "ef")) return NULL;
    CALL(thc_void_round(ctx_p, list, most, norms, scales, out, (rot_t)array_of(&g), (const float *const *)array_of(&e), st));
}

/* (handle, flat, max_norm, list, norms, workspace, stream) */
static PyObject *b_scatter_grads(ARGS)
{
    LIST_CALL(7, 3);
    double most;
    void *flat, *norms;
    if (vector(a[1], &flat, F32, sz.d, &sz, "flat") || real(a[2], &most) ||
        vector(a[4], &norms, F32, sz.n, &sz, "norms") || list_workspace(a[5], &ws, &wb, &sz)) return NULL;
    CALL(thc_scatter_grads(ctx, flat, most, list, norms, ws, wb, st));
}

/* (handle, (beta1, beta2, eps, weight_decay, max_norm), grad, list, lr, step, master, m, v, decay, norms, workspace, stream) */
static PyObject *b_adamw(ARGS)
{
    LIST_CALL(13, 3);
    thc_adamw_config cfg;
    void *grad, *lr, *step, *master, *m, *v, *decay, *norms;
    if (!PyArg_ParseTuple(a[1], "ddddd", &cfg.beta1, &cfg.beta2, &cfg.eps, &cfg.weight_decay, &cfg.max_norm)) return NULL;
    if (vector(a[2], &grad, F32, sz.d, &sz, "grad") || vector(a[4], &lr, F32, 1, &sz, "lr") ||
        vector(a[5], &step, I64, 1, &sz, "step") || vector(a[6], &master, F32, sz.d, &sz, "master") ||
        vector(a[7], &m, F32, sz.d, &sz, "m") || vector(a[8], &v, F32, sz.d, &sz, "v") ||
        vector(a[9], &decay, F32, sz.count, &sz, "decay") || vector(a[10], &norms, F32, 1, &sz, "norms") || list_workspace(a[11], &ws, &wb, &sz)) return NULL;
    CALL(thc_adamw(ctx, &cfg, grad, list, lr, step, master, m, v, decay, norms, ws, wb, st));
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))b_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    ENTRY(prepare), ENTRY(prepare_minmax), ENTRY(compress), ENTRY(prepare_compress), ENTRY(quantize_rotated),
    ENTRY(aggregate), ENTRY(decompress), ENTRY(aggregate_decompress), ENTRY(error_feedback),
    ENTRY(accumulate_error), ENTRY(prepare_noalloc), ENTRY(grad_norm), ENTRY(clip_grads), ENTRY(gather_grads),
    ENTRY(void_round), ENTRY(scatter_grads), ENTRY(adamw), {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__binding(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    if (s_data_ptr == NULL || s_nbytes == NULL || s_cuda_stream == NULL || s_dtype == NULL || s_is_contiguous == NULL ||
        s_get_device == NULL) return NULL;
    return PyModule_Create(&module);
}
