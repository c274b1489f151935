/* CPython entry to the library calls that a program makes once per layer and token.
 *
 * Marshalling only, like the ctypes binding beside it: every function takes the C call's arguments in order (device
 * pointers and the stream as integers or None) and returns its status.  A ctypes call with 14 to 18 arguments spends
 * 2 us converting them, as long as the launch itself; here it is a few nanoseconds an argument. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include "qnn.h"

static void *ptr(PyObject *o) { return o == Py_None ? NULL : PyLong_AsVoidPtr(o); }
static int64_t i64(PyObject *o) { return (int64_t)PyLong_AsLongLong(o); }
static int i32(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v > INT32_MAX || v < INT32_MIN) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit a C int");
        return 0;
    }
    return (int)v;
}
static float f32(PyObject *o) { return (float)PyFloat_AsDouble(o); }

/* every argument is converted before the call; a failed conversion leaves a Python error and nothing is called */
#define ENTRY(name, count, decl, call)                                                            \
    static PyObject *py_##name(PyObject *self, PyObject *const *a, Py_ssize_t n)                  \
    {                                                                                             \
        int status;                                                                               \
        (void)self;                                                                               \
        if (n != (count)) {                                                                       \
            PyErr_Format(PyExc_TypeError, #name " takes %d arguments, %zd given", (count), n);    \
            return NULL;                                                                          \
        }                                                                                         \
        decl;                                                                                     \
        if (PyErr_Occurred()) return NULL;                                                        \
        Py_BEGIN_ALLOW_THREADS                                                                    \
        status = call;                                                                            \
        Py_END_ALLOW_THREADS                                                                      \
        return PyLong_FromLong(status);                                                           \
    }
#define COMMA ,

ENTRY(qnn_quantize_rows_i8, 12,
      void *x = ptr(a[0]); int type = i32(a[1]); int64_t rows = i64(a[2]) COMMA K = i64(a[3]) COMMA ldx = i64(a[4]);
      void *codes = ptr(a[5]); int64_t ldq = i64(a[6]); void *scale = ptr(a[7]); void *values = ptr(a[8]);
      int vtype = i32(a[9]); int64_t ldv = i64(a[10]); void *stream = ptr(a[11]),
      qnn_quantize_rows_i8(x, type, rows, K, ldx, codes, ldq, scale, values, vtype, ldv, stream))

ENTRY(qnn_rmsnorm_quant_i8, 18,
      void *x = ptr(a[0]); void *r = ptr(a[1]); int type = i32(a[2]); int64_t rows = i64(a[3]) COMMA K = i64(a[4]) COMMA ldx = i64(a[5]) COMMA
      ldr = i64(a[6]); void *gamma = ptr(a[7]); float eps = f32(a[8]); void *codes = ptr(a[9]); int64_t ldq = i64(a[10]);
      void *scale = ptr(a[11]); void *sum = ptr(a[12]); int64_t ld_sum = i64(a[13]); void *values = ptr(a[14]); int vtype = i32(a[15]);
      int64_t ldv = i64(a[16]); void *stream = ptr(a[17]),
      qnn_rmsnorm_quant_i8(x, r, type, rows, K, ldx, ldr, gamma, eps, codes, ldq, scale, sum, ld_sum, values, vtype, ldv, stream))

ENTRY(qnn_silu_mul_quant_i8, 14,
      void *gate = ptr(a[0]); void *up = ptr(a[1]); int type = i32(a[2]); int64_t rows = i64(a[3]) COMMA K = i64(a[4]) COMMA ldg = i64(a[5]) COMMA
      ldu = i64(a[6]); void *codes = ptr(a[7]); int64_t ldq = i64(a[8]); void *scale = ptr(a[9]); void *values = ptr(a[10]);
      int vtype = i32(a[11]); int64_t ldv = i64(a[12]); void *stream = ptr(a[13]),
      qnn_silu_mul_quant_i8(gate, up, type, rows, K, ldg, ldu, codes, ldq, scale, values, vtype, ldv, stream))

ENTRY(qnn_gemm_i8_scaled, 14,
      void *x = ptr(a[0]); int64_t lda = i64(a[1]); void *sa = ptr(a[2]); void *w = ptr(a[3]); int64_t ldb = i64(a[4]); void *sb = ptr(a[5]);
      void *bias = ptr(a[6]); int64_t M = i64(a[7]) COMMA N = i64(a[8]) COMMA K = i64(a[9]); void *out = ptr(a[10]); int type = i32(a[11]);
      int64_t ldo = i64(a[12]); void *stream = ptr(a[13]),
      qnn_gemm_i8_scaled(x, lda, sa, w, ldb, sb, bias, M, N, K, out, type, ldo, stream))

ENTRY(qnn_token_logprobs, 13,
      void *z = ptr(a[0]); int type = i32(a[1]); int64_t T = i64(a[2]) COMMA V = i64(a[3]) COMMA ldl = i64(a[4]); void *ids = ptr(a[5]);
      void *lp = ptr(a[6]); void *h = ptr(a[7]); void *lse = ptr(a[8]); int topk = i32(a[9]); void *tl = ptr(a[10]); void *ti = ptr(a[11]);
      void *stream = ptr(a[12]),
      qnn_token_logprobs(z, type, T, V, ldl, ids, lp, h, lse, topk, tl, ti, stream))

ENTRY(qnn_token_logprobs_backward, 13,
      void *z = ptr(a[0]); int type = i32(a[1]); int64_t T = i64(a[2]) COMMA V = i64(a[3]) COMMA ldl = i64(a[4]); void *ids = ptr(a[5]);
      void *lse = ptr(a[6]); void *h = ptr(a[7]); void *gl = ptr(a[8]); void *gh = ptr(a[9]); void *d = ptr(a[10]); int64_t ldd = i64(a[11]);
      void *stream = ptr(a[12]),
      qnn_token_logprobs_backward(z, type, T, V, ldl, ids, lse, h, gl, gh, d, ldd, stream))

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, "status of the C call of this name"}
static PyMethodDef methods[] = {METHOD(qnn_quantize_rows_i8), METHOD(qnn_rmsnorm_quant_i8), METHOD(qnn_silu_mul_quant_i8),
                                METHOD(qnn_gemm_i8_scaled), METHOD(qnn_token_logprobs), METHOD(qnn_token_logprobs_backward),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qnn_calls", "Argument marshalling of libqnn.so calls.", -1, methods,
                                    NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__qnn_calls(void) { return PyModule_Create(&module); }
