/* Python entry points of the layer operators: marshalling only, like the ctypes binding of the other calls, but these are
 * called once per layer and step, often for a few microseconds of work, and ctypes converts a call of a dozen
 * arguments in 1.7 us where this takes 0.3.  Each function takes the C call's arguments in order, all by position
 * (addresses as ints, None = NULL), and returns its status. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/omc.h"

/* -1 in *bad if an argument is no integer in range (the exception is set).  Whatever stands for an integer is one (numpy's, say). */
static uint64_t whole(PyObject *o, int *bad)
{
    if (o == Py_None || *bad) return 0;
    PyObject *n = PyLong_Check(o) ? Py_NewRef(o) : PyNumber_Index(o);
    const unsigned long long v = n ? PyLong_AsUnsignedLongLong(n) : (unsigned long long)-1;
    Py_XDECREF(n);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) *bad = -1;
    return v;
}
static int small(PyObject *o, int *bad)
{
    if (*bad) return 0;
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) *bad = -1;
    if (v != (int)v) {
        PyErr_SetString(PyExc_OverflowError, "integer out of range");
        *bad = -1;
    }
    return (int)v;
}
static float real(PyObject *o, int *bad)
{
    if (*bad) return 0.f;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) *bad = -1;
    return (float)v;
}
static int count(Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return 1;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, got);
    return 0;
}

#define U(i) whole(a[i], &bad)
#define P(i) ((void *)(uintptr_t)whole(a[i], &bad))
#define I(i) small(a[i], &bad)
#define F(i) real(a[i], &bad)
#define ENTRY(name, n, setup, call)                                             \
    static PyObject *py_##name(PyObject *self, PyObject *const *a, Py_ssize_t got) \
    {                                                                           \
        int bad = 0, rc;                                                        \
        (void)self;                                                             \
        if (!count(got, n)) return NULL;                                        \
        setup                                                                   \
        if (bad) return NULL;                                                   \
        Py_BEGIN_ALLOW_THREADS rc = call;                                       \
        Py_END_ALLOW_THREADS return PyLong_FromLong(rc);                        \
    }

ENTRY(mx_quantise, 10,
      void *x = P(0); int type = I(1); uint64_t rows = U(2); uint64_t cols = U(3); uint64_t ld = U(4); void *codes = P(5);
      void *scales = P(6); void *codes_t = P(7); void *scales_t = P(8); void *stream = P(9);,
      omc_mx_quantise(x, type, rows, cols, ld, codes, scales, codes_t, scales_t, stream))
ENTRY(mx_dequantise, 8,
      void *codes = P(0); void *scales = P(1); uint64_t rows = U(2); uint64_t cols = U(3); void *out = P(4); int type = I(5);
      uint64_t ld = U(6); void *stream = P(7);,
      omc_mx_dequantise(codes, scales, rows, cols, out, type, ld, stream))
ENTRY(mx_matmul, 12,
      void *xc = P(0); void *xs = P(1); uint64_t m = U(2); void *wc = P(3); void *ws = P(4); uint64_t n = U(5); uint64_t k = U(6);
      void *y = P(7); int type = I(8); uint64_t ldy = U(9); void *status = P(10); void *stream = P(11);,
      omc_mx_matmul(xc, xs, m, wc, ws, n, k, y, type, ldy, status, stream))
ENTRY(mx_linear, 14,
      void *x = P(0); int type = I(1); uint64_t m = U(2); uint64_t k = U(3); uint64_t ldx = U(4); void *wc = P(5); void *ws = P(6);
      uint64_t n = U(7); void *y = P(8); int y_type = I(9); uint64_t ldy = U(10); void *space = P(11); void *status = P(12);
      void *stream = P(13);,
      omc_mx_linear(x, type, m, k, ldx, wc, ws, n, y, y_type, ldy, space, status, stream))
ENTRY(layer_norm, 13,
      void *x = P(0); int type = I(1); uint64_t rows = U(2); uint64_t cols = U(3); uint64_t ld = U(4); void *gamma = P(5);
      void *beta = P(6); float eps = F(7); void *y = P(8); uint64_t ldy = U(9); void *mean = P(10); void *rstd = P(11);
      void *stream = P(12);,
      omc_layer_norm(x, type, rows, cols, ld, gamma, beta, eps, y, ldy, mean, rstd, stream))
ENTRY(layer_norm_backward, 16,
      void *dy = P(0); uint64_t ld_dy = U(1); void *x = P(2); uint64_t ld_x = U(3); int type = I(4); uint64_t rows = U(5);
      uint64_t cols = U(6); void *gamma = P(7); void *mean = P(8); void *rstd = P(9); void *dx = P(10); uint64_t ld_dx = U(11);
      void *dgamma = P(12); void *dbeta = P(13); void *space = P(14); void *stream = P(15);,
      omc_layer_norm_backward(dy, ld_dy, x, ld_x, type, rows, cols, gamma, mean, rstd, dx, ld_dx, dgamma, dbeta, space, stream))

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, "omc_" #name ": its arguments by position; returns the status"}
static PyMethodDef methods[] = {METHOD(mx_quantise), METHOD(mx_dequantise), METHOD(mx_matmul), METHOD(mx_linear),
                                METHOD(layer_norm), METHOD(layer_norm_backward), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Entry points of libomc's layer operators.", -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
