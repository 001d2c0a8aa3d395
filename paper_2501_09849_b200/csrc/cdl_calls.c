/* Argument marshalling of the language-model calls for Python: the same five calls as in the C ABI, their addresses handed in
 * by the ctypes binding that has loaded the library.  Converting 13 to 21 arguments one by one through ctypes takes longer
 * (2.5 us) than the smallest of these calls runs on the device (1.7 us).  A pointer argument is None, an integer, or an object with
 * data_ptr(); a stream is None (the current one), an integer, or an object with cuda_stream. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "cdl.h"

static struct {
    int (*dropout)(const void *, int64_t, const void *, int64_t, void *, int64_t, int32_t, int64_t, int64_t, float, uint64_t, uint64_t, void *);
    int (*fp8_quantize)(const void *, int64_t, int32_t, int32_t, int32_t, int32_t, void *, int64_t, float *, void *, int64_t, float *, void *);
    int (*fp8_matmul)(const void *, int64_t, const float *, const void *, int64_t, const float *, int32_t, int32_t, int32_t, int32_t, void *,
                      int64_t, int32_t, const float *, void *, size_t, void *);
    int (*vocab_loss_fwd)(const void *, int64_t, const void *, int64_t, int32_t, const int64_t *, int32_t, int32_t, int32_t, float *, float *,
                          void *, size_t, void *);
    int (*vocab_loss_bwd)(const void *, int64_t, const void *, int64_t, int32_t, const int64_t *, const float *, const float *, int32_t, int32_t,
                          int32_t, void *, int64_t, void *, int64_t, void *, size_t, void *);
} fn;
static PyObject *raw_stream, *current_device;       /* callables of torch, None without a device */
static PyObject *s_data_ptr, *s_cuda_stream;

/* Each conversion leaves an exception set on failure, and the ones behind it do nothing: most of them can run Python code, which must
 * not see an exception pending.  The calls test for one before the library is entered. */
static void *ptr(PyObject *o)
{
    if (o == Py_None || PyErr_Occurred()) return NULL;
    if (PyLong_Check(o)) return (void *)(uintptr_t)PyLong_AsUnsignedLongLong(o);
    PyObject *r = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (r == NULL) return NULL;
    void *p = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(r);
    Py_DECREF(r);
    return p;
}
static void *stream(PyObject *o)
{
    if (PyErr_Occurred()) return NULL;
    if (o == Py_None) {
        if (raw_stream == NULL || raw_stream == Py_None) return NULL;
        PyObject *d = PyObject_CallNoArgs(current_device);
        if (d == NULL) return NULL;
        PyObject *r = PyObject_CallOneArg(raw_stream, d);
        Py_DECREF(d);
        if (r == NULL) return NULL;
        void *p = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(r);
        Py_DECREF(r);
        return p;
    }
    if (PyLong_Check(o)) return (void *)(uintptr_t)PyLong_AsUnsignedLongLong(o);
    PyObject *r = PyObject_GetAttr(o, s_cuda_stream);
    if (r == NULL) return NULL;
    void *p = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(r);
    Py_DECREF(r);
    return p;
}
static int64_t i64(PyObject *o) { return PyErr_Occurred() ? 0 : (int64_t)PyLong_AsLongLong(o); }
static uint64_t u64(PyObject *o) { return PyErr_Occurred() ? 0 : (uint64_t)PyLong_AsUnsignedLongLongMask(o); }
static double f64(PyObject *o) { return PyErr_Occurred() ? 0.0 : PyFloat_AsDouble(o); }
static int32_t i32(PyObject *o)
{
    if (PyErr_Occurred()) return 0;
    const long v = PyLong_AsLong(o);
    if ((v > INT32_MAX || v < INT32_MIN) && !PyErr_Occurred()) PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
    return (int32_t)v;
}
static int ready(const void *f, Py_ssize_t n, Py_ssize_t want)
{
    if (f == NULL) PyErr_SetString(PyExc_RuntimeError, "the library is not loaded");
    else if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments wanted, %zd given", want, n);
    else return 1;
    return 0;
}
#define ARGS PyObject *self, PyObject *const *a, Py_ssize_t n
/* (a launch can wait for room in the device's queue: other threads run meanwhile) */
#define FINISH(call)                       \
    do {                                   \
        int rc;                            \
        if (PyErr_Occurred()) return NULL; \
        Py_BEGIN_ALLOW_THREADS             \
        rc = call;                         \
        Py_END_ALLOW_THREADS               \
        return PyLong_FromLong((long)rc);  \
    } while (0)

static PyObject *py_dropout(ARGS)
{
    (void)self;
    if (!ready((const void *)(uintptr_t)fn.dropout, n, 13)) return NULL;
    const void *x = ptr(a[0]), *res = ptr(a[2]);
    void *y = ptr(a[4]), *st = stream(a[12]);
    const int64_t ldx = i64(a[1]), ldr = i64(a[3]), ldy = i64(a[5]), rows = i64(a[7]), cols = i64(a[8]);
    const int32_t type = i32(a[6]);
    const double p = f64(a[9]);
    const uint64_t seed = u64(a[10]), first = u64(a[11]);
    FINISH(fn.dropout(x, ldx, res, ldr, y, ldy, type, rows, cols, (float)p, seed, first, st));
}

static PyObject *py_fp8_quantize(ARGS)
{
    (void)self;
    if (!ready((const void *)(uintptr_t)fn.fp8_quantize, n, 13)) return NULL;
    const void *x = ptr(a[0]);
    const int64_t ldx = i64(a[1]), ldc = i64(a[7]), ldt = i64(a[10]);
    const int32_t type = i32(a[2]), rows = i32(a[3]), cols = i32(a[4]), mode = i32(a[5]);
    void *codes = ptr(a[6]), *codes_t = ptr(a[9]), *st = stream(a[12]);
    float *scales = ptr(a[8]), *scales_t = ptr(a[11]);
    FINISH(fn.fp8_quantize(x, ldx, type, rows, cols, mode, codes, ldc, scales, codes_t, ldt, scales_t, st));
}

static PyObject *py_fp8_matmul(ARGS)
{
    (void)self;
    if (!ready((const void *)(uintptr_t)fn.fp8_matmul, n, 17)) return NULL;
    const void *A = ptr(a[0]), *B = ptr(a[3]);
    const float *sa = ptr(a[2]), *sb = ptr(a[5]), *bias = ptr(a[13]);
    const int64_t lda = i64(a[1]), ldb = i64(a[4]), ldo = i64(a[11]), bytes = i64(a[15]);
    const int32_t mode = i32(a[6]), M = i32(a[7]), N = i32(a[8]), K = i32(a[9]), type = i32(a[12]);
    void *out = ptr(a[10]), *ws = ptr(a[14]), *st = stream(a[16]);
    FINISH(fn.fp8_matmul(A, lda, sa, B, ldb, sb, mode, M, N, K, out, ldo, type, bias, ws, (size_t)(bytes < 0 ? 0 : bytes), st));
}

static PyObject *py_vocab_loss_fwd(ARGS)
{
    (void)self;
    if (!ready((const void *)(uintptr_t)fn.vocab_loss_fwd, n, 14)) return NULL;
    const void *H = ptr(a[0]), *W = ptr(a[2]);
    const int64_t ldh = i64(a[1]), ldw = i64(a[3]), bytes = i64(a[12]);
    const int64_t *labels = ptr(a[5]);
    const int32_t type = i32(a[4]), T = i32(a[6]), V = i32(a[7]), D = i32(a[8]);
    float *loss = ptr(a[9]), *lse = ptr(a[10]);
    void *ws = ptr(a[11]), *st = stream(a[13]);
    FINISH(fn.vocab_loss_fwd(H, ldh, W, ldw, type, labels, T, V, D, loss, lse, ws, (size_t)(bytes < 0 ? 0 : bytes), st));
}

static PyObject *py_vocab_loss_bwd(ARGS)
{
    (void)self;
    if (!ready((const void *)(uintptr_t)fn.vocab_loss_bwd, n, 18)) return NULL;
    const void *H = ptr(a[0]), *W = ptr(a[2]);
    const int64_t ldh = i64(a[1]), ldw = i64(a[3]), lddh = i64(a[12]), lddw = i64(a[14]), bytes = i64(a[16]);
    const int64_t *labels = ptr(a[5]);
    const float *lse = ptr(a[6]), *dloss = ptr(a[7]);
    const int32_t type = i32(a[4]), T = i32(a[8]), V = i32(a[9]), D = i32(a[10]);
    void *dH = ptr(a[11]), *dW = ptr(a[13]), *ws = ptr(a[15]), *st = stream(a[17]);
    FINISH(fn.vocab_loss_bwd(H, ldh, W, ldw, type, labels, lse, dloss, T, V, D, dH, lddh, dW, lddw, ws, (size_t)(bytes < 0 ? 0 : bytes), st));
}

/* bind(raw stream getter, device getter, addresses of the five calls) */
static PyObject *py_bind(ARGS)
{
    (void)self;
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "7 arguments wanted");
        return NULL;
    }
    uintptr_t at[5];
    for (int i = 0; i < 5; ++i) at[i] = (uintptr_t)PyLong_AsUnsignedLongLong(a[2 + i]);
    if (PyErr_Occurred()) return NULL;
    Py_INCREF(a[0]);
    Py_XSETREF(raw_stream, a[0]);
    Py_INCREF(a[1]);
    Py_XSETREF(current_device, a[1]);
    *(void **)&fn.dropout = (void *)at[0];
    *(void **)&fn.fp8_quantize = (void *)at[1];
    *(void **)&fn.fp8_matmul = (void *)at[2];
    *(void **)&fn.vocab_loss_fwd = (void *)at[3];
    *(void **)&fn.vocab_loss_bwd = (void *)at[4];
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind), METHOD(dropout), METHOD(fp8_quantize), METHOD(fp8_matmul), METHOD(vocab_loss_fwd), METHOD(vocab_loss_bwd),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cdl_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__cdl_calls(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (s_data_ptr == NULL || s_cuda_stream == NULL) return NULL;
    return PyModule_Create(&module);
}
