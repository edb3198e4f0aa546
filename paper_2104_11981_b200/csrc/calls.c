/* CPython entry points of the training operators' calls: numbers in, status code out, nothing else.  ctypes takes 1.9
 * to 2.5 us to convert the 16 to 22 arguments of these calls, as long as the launch itself; this takes 0.2. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <limits.h>
#include <stdint.h>

#include "decentlam.h"

/* Whole numbers and addresses; None is 0. */
static int64_t whole(PyObject* o) { return o == Py_None ? 0 : (int64_t)PyLong_AsLongLong(o); }
/* An int parameter: held to its range, so that what is too large stays so. */
static int held(int64_t v) { return v > INT_MAX ? INT_MAX : v < INT_MIN ? INT_MIN : (int)v; }

#define N(k) whole(args[k])
#define I(k) held(whole(args[k]))
#define P(k) ((void*)(uintptr_t)whole(args[k]))
#define F(k) ((float)PyFloat_AsDouble(args[k]))

#define CALL(name, count, ...)                                                                              \
    static PyObject* py_##name(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {                   \
        int status;                                                                                         \
        (void)self;                                                                                         \
        if (nargs != count) return PyErr_Format(PyExc_TypeError, #name ": %d arguments expected", count);   \
        __VA_ARGS__;                                                                                        \
        return PyLong_FromLong(status);                                                                     \
    }
/* Converts first: what does not convert raises before the call.  The call itself runs without the interpreter's lock. */
#define LAUNCH(call)                       \
    if (PyErr_Occurred()) return NULL;     \
    Py_BEGIN_ALLOW_THREADS status = call;  \
    Py_END_ALLOW_THREADS

CALL(gradient_norm, 4, {
    dlm_gradients* list = P(0);
    int kind = I(1);
    float* norms = P(2);
    void* stream = P(3);
    LAUNCH(gradient_norm(list, kind, norms, stream))
})

CALL(gradient_clip, 8, {
    dlm_gradients* list = P(0);
    int kind = I(1), g_dtype = I(5);
    float max_norm = F(2);
    float* norms = P(3);
    void *g = P(4), *stream = P(7);
    int64_t ldg = N(6);
    LAUNCH(gradient_clip(list, kind, max_norm, norms, g, g_dtype, ldg, stream))
})

CALL(layer_norm, 16, {
    int n = I(0), dtype = I(4);
    int64_t rows = N(1), c = N(2), ldx = N(5), ldw = N(7), ldb = N(9), ldy = N(12);
    void *x = P(3), *w = P(6), *b = P(8), *y = P(11), *mean = P(13), *rstd = P(14), *stream = P(15);
    float eps = F(10);
    LAUNCH(layer_norm(n, rows, c, x, dtype, ldx, w, ldw, b, ldb, eps, y, ldy, mean, rstd, stream))
})

CALL(layer_norm_grad, 22, {
    int n = I(0), dtype = I(4), g_dtype = I(18);
    int64_t rows = N(1), c = N(2), ldx = N(5), lddy = N(7), ldw = N(9), lddx = N(13), ldgw = N(15), ldgb = N(17), bytes = N(20);
    void *x = P(3), *dy = P(6), *w = P(8), *mean = P(10), *rstd = P(11), *dx = P(12), *gw = P(14), *gb = P(16), *work = P(19),
         *stream = P(21);
    LAUNCH(layer_norm_grad(n, rows, c, x, dtype, ldx, dy, lddy, w, ldw, mean, rstd, dx, lddx, gw, ldgw, gb, ldgb, g_dtype, work,
                           bytes, stream))
})

CALL(policy_loss_grad, 21, {
    int n = I(0), dtype = I(4);
    int64_t rows = N(1), vocab = N(2), ldl = N(5), ldd = N(17), bytes = N(19);
    void *z = P(3), *tokens = P(6), *w = P(7), *adv = P(8), *old = P(9), *ref = P(10), *loss = P(14), *logp = P(15), *d = P(16),
         *work = P(18), *stream = P(20);
    float lo = F(11), hi = F(12), kl = F(13);
    LAUNCH(policy_loss_grad(n, rows, vocab, z, dtype, ldl, tokens, w, adv, old, ref, lo, hi, kl, loss, logp, d, ldd, work, bytes,
                            stream))
})

CALL(embedding, 13, {
    int n = I(0), t_dtype = I(5), dtype = I(10);
    int64_t rows = N(1), vocab = N(2), c = N(3), ldt = N(6), ldy = N(11);
    void *table = P(4), *tokens = P(7), *y = P(9), *stream = P(12);
    float scale = F(8);
    LAUNCH(embedding(n, rows, vocab, c, table, t_dtype, ldt, tokens, scale, y, dtype, ldy, stream))
})

CALL(embedding_grad, 16, {
    int n = I(0), dtype = I(6), accumulate = I(9), g_dtype = I(11);
    int64_t rows = N(1), vocab = N(2), c = N(3), lddy = N(7), ldgt = N(12), bytes = N(14);
    void *tokens = P(4), *dy = P(5), *dtable = P(10), *work = P(13), *stream = P(15);
    float scale = F(8);
    LAUNCH(embedding_grad(n, rows, vocab, c, tokens, dy, dtype, lddy, scale, accumulate, dtable, g_dtype, ldgt, work, bytes, stream))
})

CALL(rms_norm, 20, {
    int n = I(0), dtype = I(4);
    int64_t rows = N(1), c = N(2), ldx = N(5), ldr = N(7), ldw = N(9), ldh = N(12), ldy = N(14), ld8 = N(16);
    void *x = P(3), *res = P(6), *w = P(8), *h = P(11), *y = P(13), *y8 = P(15), *scales = P(17), *rstd = P(18), *stream = P(19);
    float eps = F(10);
    LAUNCH(rms_norm(n, rows, c, x, dtype, ldx, res, ldr, w, ldw, eps, h, ldh, y, ldy, y8, ld8, scales, rstd, stream))
})

CALL(rms_norm_grad, 21, {
    int n = I(0), dtype = I(4), g_dtype = I(17);
    int64_t rows = N(1), c = N(2), ldh = N(5), lddy = N(7), lddr = N(9), ldw = N(11), lddh = N(14), ldgw = N(16), bytes = N(19);
    void *h = P(3), *dy = P(6), *dres = P(8), *w = P(10), *rstd = P(12), *dh = P(13), *gw = P(15), *work = P(18), *stream = P(20);
    LAUNCH(rms_norm_grad(n, rows, c, h, dtype, ldh, dy, lddy, dres, lddr, w, ldw, rstd, dh, lddh, gw, ldgw, g_dtype, work, bytes,
                         stream))
})

CALL(dropout, 14, {
    int n = I(0), dtype = I(4);
    int64_t rows = N(1), c = N(2), ldx = N(5), ldr = N(7), site = N(10), ldy = N(12);
    void *x = P(3), *res = P(6), *state = P(9), *y = P(11), *stream = P(13);
    float p = F(8);
    LAUNCH(dropout(n, rows, c, x, dtype, ldx, res, ldr, p, state, site, y, ldy, stream))
})

CALL(logits_adjust, 20, {
    int n = I(0), dtype = I(4);
    int64_t rows = N(1), vocab = N(2), ldl = N(5), ldb = N(7), ldm = N(9), length = N(11), ldo = N(18);
    void *z = P(3), *bias = P(6), *allowed = P(8), *text = P(10), *start = P(12), *rep = P(13), *freq = P(14), *pres = P(15),
         *temp = P(16), *out = P(17), *stream = P(19);
    LAUNCH(logits_adjust(n, rows, vocab, z, dtype, ldl, bias, ldb, allowed, ldm, text, length, start, rep, freq, pres, temp, out, ldo,
                         stream))
})

CALL(logits_adjust_grad, 18, {
    int n = I(0), dtype = I(4);
    int64_t rows = N(1), vocab = N(2), lddo = N(5), ldl = N(7), ldm = N(9), length = N(11), ldd = N(16);
    void *g = P(3), *z = P(6), *allowed = P(8), *text = P(10), *start = P(12), *rep = P(13), *temp = P(14), *d = P(15),
         *stream = P(17);
    LAUNCH(logits_adjust_grad(n, rows, vocab, g, dtype, lddo, z, ldl, allowed, ldm, text, length, start, rep, temp, d, ldd, stream))
})

/* The operators between tokens and logits with tensors themselves as arguments, read through the DLPack exchange interface (a struct of C
 * functions that the tensors' class offers as a capsule): a call on a single token costs what its launch costs.  The checks are those of
 * binding.py, which makes them itself where the interface is missing. */
#ifdef DLM_TENSORS
#include <ATen/dlpack.h>

static const DLPackExchangeAPI* exchange;
static PyTypeObject* tensor_type;

static PyObject* py_read_tensors(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    (void)self;
    if (nargs != 2 || !PyType_Check(args[0])) return PyErr_Format(PyExc_TypeError, "read_tensors: the tensors' type and its capsule");
    const DLPackExchangeAPI* api = PyCapsule_GetPointer(args[1], "dlpack_exchange_api");
    if (!api) return NULL;
    while (api && api->header.version.major != DLPACK_MAJOR_VERSION) api = (const DLPackExchangeAPI*)api->header.prev_api;
    if (!api || !api->dltensor_from_py_object_no_sync || !api->current_work_stream) Py_RETURN_FALSE;
    Py_INCREF(args[0]);
    tensor_type = (PyTypeObject*)args[0];
    exchange = api;
    Py_RETURN_TRUE;
}

typedef struct {
    DLTensor t;
    char* data; /* NULL: None */
} Tensor;
enum { F32 = DLM_G_F32, BF16 = DLM_G_BF16, ANY = -1, I64 = -2, I32 = -3, E4M3 = -4, BYTES = -5 };
static int kind_of(const Tensor* x) {
    const DLDataType d = x->t.dtype;
    if (d.lanes != 1) return ANY - 100;
    if (d.code == kDLFloat && d.bits == 32) return F32;
    if (d.code == kDLBfloat && d.bits == 16) return BF16;
    if (d.code == kDLInt && d.bits == 64) return I64;
    if (d.code == kDLInt && d.bits == 32) return I32;
    if (d.code == kDLFloat8_e4m3fn && d.bits == 8) return E4M3;
    return ANY - 100;
}
#define FAIL(...) return PyErr_Format(PyExc_AssertionError, __VA_ARGS__), 0
/* A tensor of this kind on the current device, or None where that is allowed. */
static int tensor(PyObject* o, long home, int kind, int none, Tensor* x) {
    x->data = NULL;
    if (o == Py_None && none) return 1;
    if (!PyObject_TypeCheck(o, tensor_type)) return PyErr_Format(PyExc_TypeError, "a tensor is expected"), 0;
    if (exchange->dltensor_from_py_object_no_sync(o, &x->t) != 0) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "this tensor cannot be read");
        return 0;
    }
    if (x->t.device.device_type != kDLCUDA || x->t.device.device_id != home) FAIL("tensors on the current CUDA device are expected");
    if (kind == ANY) {
        if (kind_of(x) < 0) return PyErr_Format(PyExc_TypeError, "float32 or bfloat16 expected"), 0;
    } else if (kind != BYTES && kind_of(x) != kind) {
        FAIL("a tensor of another type is expected");
    }
    x->data = (char*)x->t.data + x->t.byte_offset;
    return 1;
}
static int contiguous(const Tensor* x) {
    int64_t want = 1;
    if (!x->t.strides) return 1;
    for (int k = 0; k < x->t.ndim; ++k)
        if (x->t.shape[k] == 0) return 1;
    for (int k = x->t.ndim - 1; k >= 0; --k) {
        if (x->t.shape[k] != 1 && x->t.strides[k] != want) return 0;
        want *= x->t.shape[k];
    }
    return 1;
}
static int64_t count_of(const Tensor* x) {
    int64_t n = 1;
    for (int k = 0; k < x->t.ndim; ++k) n *= x->t.shape[k];
    return n;
}
/* Row stride of [n, rows, c], whose nodes follow one another. */
static int rows_of(const Tensor* x, const int64_t* shape, int64_t* ld) {
    if (x->t.ndim != 3 || x->t.shape[0] != shape[0] || x->t.shape[1] != shape[1] || x->t.shape[2] != shape[2])
        FAIL("a tensor of the same shape is expected");
    if (contiguous(x)) return *ld = shape[2], 1;
    const int64_t* s = x->t.strides;
    if (s[2] != 1 && shape[2] != 1) FAIL("unit column stride expected");
    if (shape[1] == 1) return *ld = s[0], 1;
    if (shape[0] != 1 && s[0] != shape[1] * s[1]) FAIL("the nodes' rows must be evenly spaced");
    return *ld = s[1], 1;
}
static int rows(PyObject* o, long home, int kind, int none, const int64_t* shape, Tensor* x, int64_t* ld) {
    if (!tensor(o, home, kind, none, x)) return 0;
    if (o == Py_None) return *ld = 0, 1;
    return rows_of(x, shape, ld);
}
static int vectors(PyObject* o, long home, int kind, int none, int64_t n, int64_t c, Tensor* x, int64_t* ld) {
    *ld = 0;
    if (!tensor(o, home, kind, none, x)) return 0;
    if (o == Py_None) return 1;
    if (x->t.ndim != 2 || x->t.shape[0] != n || x->t.shape[1] != c) FAIL("per-node vectors [n, c] are expected");
    if (x->t.strides && x->t.strides[1] != 1 && c != 1) FAIL("unit column stride expected");
    *ld = n > 1 && x->t.strides ? x->t.strides[0] : c;
    return 1;
}
static int flat(PyObject* o, long home, int kind, int none, int64_t count, Tensor* x) {
    if (!tensor(o, home, kind, none, x)) return 0;
    if (o == Py_None) return 1;
    if ((count >= 0 && count_of(x) != count) || !contiguous(x)) FAIL("a contiguous tensor of another length is expected");
    return 1;
}
static int tables(PyObject* o, long home, Tensor* x, int64_t* ld) {
    if (!tensor(o, home, ANY, 0, x)) return 0;
    if (x->t.ndim != 3) FAIL("tables [n, vocab, c] are expected");
    const int64_t *z = x->t.shape, *s = x->t.strides;
    if (s && ((s[2] != 1 && z[2] != 1) || (s[1] != z[2] && z[1] != 1))) FAIL("a node's rows follow one another");
    *ld = z[0] > 1 && s ? s[0] : z[1] * z[2];
    return 1;
}
static int shape3(const Tensor* x) {
    if (x->t.ndim != 3) FAIL("[n, rows, c] is expected");
    return 1;
}
static int64_t bytes_of(const Tensor* x) { return count_of(x) * ((x->t.dtype.bits * x->t.dtype.lanes + 7) / 8); }
static int on_stream(PyObject* o, long home, void** stream) {
    if (o != Py_None) return *stream = (void*)(uintptr_t)PyLong_AsUnsignedLongLong(o), !PyErr_Occurred();
    if (exchange->current_work_stream(kDLCUDA, (int32_t)home, stream) != 0) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "no current stream");
        return 0;
    }
    return 1;
}
/* The last two arguments are the current device and the stream (None: the current one). */
#define TENSOR_CALL(name, count, ...)                                                                                      \
    static PyObject* py_##name##_of(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {                             \
        int status;                                                                                                        \
        void* stream;                                                                                                      \
        (void)self;                                                                                                        \
        if (nargs != count + 2 || !exchange) return PyErr_Format(PyExc_TypeError, #name ": %d arguments expected", count); \
        const long home = PyLong_AsLong(args[count]);                                                                      \
        if (!on_stream(args[count + 1], home, &stream)) return NULL;                                                       \
        __VA_ARGS__                                                                                                        \
        return PyLong_FromLong(status);                                                                                    \
    }
#define NEED(what) \
    if (!(what)) return NULL

TENSOR_CALL(embedding, 4, {
    Tensor table, tokens, y;
    int64_t ldt, ldy;
    const float scale = F(3);
    NEED(tables(args[0], home, &table, &ldt) && tensor(args[2], home, ANY, 0, &y) && shape3(&y));
    const int64_t *z = table.t.shape, want[3] = {z[0], y.t.shape[1], z[2]};
    NEED(rows_of(&y, want, &ldy) && flat(args[1], home, I64, 0, want[0] * want[1], &tokens));
    LAUNCH(embedding(held(z[0]), want[1], z[1], z[2], table.data, kind_of(&table), ldt, (void*)tokens.data, scale, y.data, kind_of(&y),
                     ldy, stream))
})

TENSOR_CALL(embedding_grad, 6, {
    Tensor tokens, dy, table, work;
    int64_t ldt, ldy;
    const float scale = F(4);
    const int accumulate = PyObject_IsTrue(args[5]);
    NEED(tables(args[2], home, &table, &ldt) && tensor(args[1], home, ANY, 0, &dy) && shape3(&dy));
    const int64_t *z = table.t.shape, want[3] = {z[0], dy.t.shape[1], z[2]};
    NEED(rows_of(&dy, want, &ldy) && flat(args[0], home, I64, 0, want[0] * want[1], &tokens) &&
         flat(args[3], home, BYTES, 0, -1, &work));
    LAUNCH(embedding_grad(held(z[0]), want[1], z[1], z[2], (void*)tokens.data, dy.data, kind_of(&dy), ldy, scale, accumulate,
                          table.data, kind_of(&table), ldt, work.data, bytes_of(&work), stream))
})

TENSOR_CALL(rms_norm, 9, {
    Tensor x, w, y, rstd, res, h, y8, scales;
    int64_t ldx, ldw, ldy, ldr, ldh, ld8;
    const float eps = F(2);
    NEED(tensor(args[0], home, ANY, 0, &x) && shape3(&x));
    const int64_t* z = x.t.shape;
    const int kind = kind_of(&x);
    NEED(rows_of(&x, z, &ldx) && vectors(args[1], home, F32, 0, z[0], z[2], &w, &ldw) && rows(args[3], home, kind, 1, z, &y, &ldy) &&
         flat(args[4], home, F32, 0, z[0] * z[1], &rstd) && rows(args[5], home, kind, 1, z, &res, &ldr) &&
         rows(args[6], home, kind, 1, z, &h, &ldh) && rows(args[7], home, E4M3, 1, z, &y8, &ld8) &&
         flat(args[8], home, F32, 1, z[0] * z[1], &scales));
    LAUNCH(rms_norm(held(z[0]), z[1], z[2], x.data, kind, ldx, res.data, ldr, (void*)w.data, ldw, eps, h.data, ldh, y.data, ldy,
                    y8.data, ld8, (void*)scales.data, (void*)rstd.data, stream))
})

TENSOR_CALL(rms_norm_grad, 8, {
    Tensor h, dy, w, rstd, dh, dw, work, res;
    int64_t ldh, lddy, ldw, lddh, ldgw, ldr;
    NEED(tensor(args[0], home, ANY, 0, &h) && shape3(&h));
    const int64_t* z = h.t.shape;
    const int kind = kind_of(&h);
    NEED(rows_of(&h, z, &ldh) && rows(args[1], home, kind, 0, z, &dy, &lddy) && vectors(args[2], home, F32, 0, z[0], z[2], &w, &ldw) &&
         flat(args[3], home, F32, 0, z[0] * z[1], &rstd) && rows(args[4], home, kind, 0, z, &dh, &lddh) &&
         vectors(args[5], home, ANY, 0, z[0], z[2], &dw, &ldgw) && flat(args[6], home, BYTES, 0, -1, &work) &&
         rows(args[7], home, kind, 1, z, &res, &ldr));
    LAUNCH(rms_norm_grad(held(z[0]), z[1], z[2], h.data, kind, ldh, dy.data, lddy, res.data, ldr, (void*)w.data, ldw,
                         (void*)rstd.data, dh.data, lddh, dw.data, ldgw, kind_of(&dw), work.data, bytes_of(&work), stream))
})

TENSOR_CALL(dropout, 6, {
    Tensor x, state, y, res;
    int64_t ldx, ldy, ldr;
    const float p = F(1);
    const int64_t site = N(4);
    NEED(tensor(args[0], home, ANY, 0, &x) && shape3(&x));
    const int64_t* z = x.t.shape;
    const int kind = kind_of(&x);
    NEED(rows_of(&x, z, &ldx) && flat(args[2], home, I64, 0, 2, &state) && rows(args[3], home, kind, 0, z, &y, &ldy) &&
         rows(args[5], home, kind, 1, z, &res, &ldr));
    LAUNCH(dropout(held(z[0]), z[1], z[2], x.data, kind, ldx, res.data, ldr, p, (void*)state.data, site, y.data, ldy, stream))
})

/* A bit mask [n, rows, words]; expanded from one row: 0 words between rows. */
static int mask(PyObject* o, long home, const int64_t* z, Tensor* x, int64_t* ld) {
    *ld = 0;
    if (!tensor(o, home, I32, 1, x)) return 0;
    if (o == Py_None) return 1;
    if (x->t.ndim != 3 || x->t.shape[0] != z[0] || x->t.shape[1] != z[1] || x->t.shape[2] < (z[2] + 31) / 32)
        FAIL("a bit for each token of each row is expected");
    if (!contiguous(x) && x->t.strides[0] == 0 && x->t.strides[1] == 0) {
        if (x->t.strides[2] != 1 && x->t.shape[2] != 1) FAIL("unit stride of the words is expected");
        return 1;
    }
    return rows_of(x, x->t.shape, ld);
}
static int texts(PyObject* text, PyObject* start, long home, int64_t count, Tensor* t, Tensor* s, int64_t* length) {
    *length = 0;
    if (!flat(text, home, I64, 1, -1, t) || !flat(start, home, I64, 1, count + 1, s)) return 0;
    if ((text == Py_None) != (start == Py_None)) FAIL("a text and its bounds are expected");
    if (text != Py_None) *length = count_of(t);
    return 1;
}

TENSOR_CALL(logits_adjust, 10, {
    Tensor in, out, bias, allowed, text, start, rep, freq, pres, temp;
    int64_t ldl, ldo, ldb, ldm, length;
    NEED(tensor(args[0], home, ANY, 0, &in) && shape3(&in));
    const int64_t *z = in.t.shape, count = z[0] * z[1];
    const int kind = kind_of(&in);
    NEED(rows_of(&in, z, &ldl) && rows(args[1], home, kind, 0, z, &out, &ldo) &&
         vectors(args[2], home, F32, 1, z[0], z[2], &bias, &ldb) &&
         mask(args[3], home, z, &allowed, &ldm) && texts(args[4], args[5], home, count, &text, &start, &length) &&
         flat(args[6], home, F32, 1, count, &rep) && flat(args[7], home, F32, 1, count, &freq) &&
         flat(args[8], home, F32, 1, count, &pres) && flat(args[9], home, F32, 1, count, &temp));
    LAUNCH(logits_adjust(held(z[0]), z[1], z[2], in.data, kind, ldl, (void*)bias.data, ldb, (void*)allowed.data, ldm,
                         (void*)text.data, length, (void*)start.data, (void*)rep.data, (void*)freq.data, (void*)pres.data,
                         (void*)temp.data, out.data, ldo, stream))
})

TENSOR_CALL(logits_adjust_grad, 8, {
    Tensor d, out, in, allowed, text, start, rep, temp;
    int64_t ldd, ldo, ldl, ldm, length;
    NEED(tensor(args[0], home, ANY, 0, &d) && shape3(&d));
    const int64_t *z = d.t.shape, count = z[0] * z[1];
    const int kind = kind_of(&d);
    NEED(rows_of(&d, z, &ldd) && rows(args[1], home, kind, 0, z, &out, &ldo) && rows(args[2], home, kind, 1, z, &in, &ldl) &&
         mask(args[3], home, z, &allowed, &ldm) && texts(args[4], args[5], home, count, &text, &start, &length) &&
         flat(args[6], home, F32, 1, count, &rep) && flat(args[7], home, F32, 1, count, &temp));
    LAUNCH(logits_adjust_grad(held(z[0]), z[1], z[2], d.data, kind, ldd, in.data, ldl, (void*)allowed.data, ldm, (void*)text.data,
                              length, (void*)start.data, (void*)rep.data, (void*)temp.data, out.data, ldo, stream))
})
#endif

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {ENTRY(gradient_norm), ENTRY(gradient_clip), ENTRY(layer_norm), ENTRY(layer_norm_grad),
                                ENTRY(policy_loss_grad), ENTRY(embedding), ENTRY(embedding_grad), ENTRY(rms_norm),
                                ENTRY(rms_norm_grad), ENTRY(dropout), ENTRY(logits_adjust), ENTRY(logits_adjust_grad),
#ifdef DLM_TENSORS
                                ENTRY(read_tensors), ENTRY(embedding_of), ENTRY(embedding_grad_of), ENTRY(rms_norm_of),
                                ENTRY(rms_norm_grad_of), ENTRY(dropout_of), ENTRY(logits_adjust_of), ENTRY(logits_adjust_grad_of),
#endif
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
