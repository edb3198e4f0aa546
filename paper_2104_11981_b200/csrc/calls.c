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

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {ENTRY(gradient_norm), ENTRY(gradient_clip), ENTRY(layer_norm), ENTRY(layer_norm_grad),
                                ENTRY(policy_loss_grad), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
