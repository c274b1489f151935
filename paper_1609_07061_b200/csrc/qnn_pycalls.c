/* CPython entry to the library calls that a program makes once per layer and token.
 *
 * Marshalling only, like the ctypes binding beside it: every function takes the C call's arguments in order, with tensors
 * where the C call takes device pointers (their types are checked, and give the call's type arguments), and returns its
 * status.  ctypes spends 2 us on 14 to 18 arguments, and checking eight tensors in Python another 1 us, as long as the
 * launch itself; here an argument costs a few and a tensor some 50 nanoseconds. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include "qnn.h"

static PyObject *s_dtype, *s_data_ptr;                   /* attribute names */
static PyObject *t_f32, *t_bf16, *t_f16, *t_i8, *t_i64;  /* torch's type objects: one of each exists */

static void *ptr(PyObject *o) { return o == Py_None ? NULL : PyLong_AsVoidPtr(o); }
/* pointer of a tensor of any type; None gives NULL */
static void *any(PyObject *t)
{
    void *p;
    PyObject *v;
    if (t == Py_None || PyErr_Occurred()) return NULL;
    v = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (v == NULL) return NULL;
    p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return p;
}
/* pointer of a tensor of one type */
static void *need(PyObject *t, PyObject *dtype, const char *where)
{
    PyObject *d;
    if (t == Py_None || PyErr_Occurred()) return NULL;
    d = PyObject_GetAttr(t, s_dtype);
    if (d == NULL) return NULL;
    Py_DECREF(d);                                        /* (a type object outlives its tensors) */
    if (d != dtype) {
        PyErr_Format(PyExc_TypeError, "%s: %S where %S is needed", where, d, dtype);
        return NULL;
    }
    return any(t);
}
/* type object of a real tensor and its QNN_TYPE_*; None counts as float32 */
static PyObject *real(PyObject *t, int *type, const char *where)
{
    PyObject *d;
    *type = QNN_TYPE_F32;
    if (t == Py_None || PyErr_Occurred()) return t_f32;
    d = PyObject_GetAttr(t, s_dtype);
    if (d == NULL) return t_f32;
    Py_DECREF(d);
    if (d == t_bf16) *type = QNN_TYPE_BF16;
    else if (d == t_f16) *type = QNN_TYPE_F16;
    else if (d != t_f32) PyErr_Format(PyExc_TypeError, "%s: %S where float32, bfloat16 or float16 is needed", where, d);
    return d;
}
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

ENTRY(qnn_quantize_rows_i8, 10,
      const char *w = "qnn_quantize_rows_i8"; int type COMMA vtype = QNN_TYPE_F32; real(a[0], &type, w);
      void *x = any(a[0]); int64_t rows = i64(a[1]) COMMA K = i64(a[2]) COMMA ldx = i64(a[3]);
      void *codes = need(a[4], t_i8, w); int64_t ldq = i64(a[5]); void *scale = need(a[6], t_f32, w); real(a[7], &vtype, w);
      void *values = any(a[7]); int64_t ldv = i64(a[8]); void *stream = ptr(a[9]),
      qnn_quantize_rows_i8(x, type, rows, K, ldx, codes, ldq, scale, values, vtype, ldv, stream))

ENTRY(qnn_rmsnorm_quant_i8, 16,
      const char *w = "qnn_rmsnorm_quant_i8"; int type COMMA vtype; PyObject *dt = real(a[0], &type, w);
      void *x = any(a[0]); void *r = need(a[1], dt, w); int64_t rows = i64(a[2]) COMMA K = i64(a[3]) COMMA ldx = i64(a[4]) COMMA
      ldr = i64(a[5]); void *gamma = need(a[6], dt, w); float eps = f32(a[7]); void *codes = need(a[8], t_i8, w); int64_t ldq = i64(a[9]);
      void *scale = need(a[10], t_f32, w); void *sum = need(a[11], dt, w); int64_t ld_sum = i64(a[12]); real(a[13], &vtype, w);
      void *values = any(a[13]); int64_t ldv = i64(a[14]); void *stream = ptr(a[15]),
      qnn_rmsnorm_quant_i8(x, r, type, rows, K, ldx, ldr, gamma, eps, codes, ldq, scale, sum, ld_sum, values, vtype, ldv, stream))

ENTRY(qnn_silu_mul_quant_i8, 12,
      const char *w = "qnn_silu_mul_quant_i8"; int type COMMA vtype; PyObject *dt = real(a[0], &type, w);
      void *gate = any(a[0]); void *up = need(a[1], dt, w); int64_t rows = i64(a[2]) COMMA K = i64(a[3]) COMMA ldg = i64(a[4]) COMMA
      ldu = i64(a[5]); void *codes = need(a[6], t_i8, w); int64_t ldq = i64(a[7]); void *scale = need(a[8], t_f32, w); real(a[9], &vtype, w);
      void *values = any(a[9]); int64_t ldv = i64(a[10]); void *stream = ptr(a[11]),
      qnn_silu_mul_quant_i8(gate, up, type, rows, K, ldg, ldu, codes, ldq, scale, values, vtype, ldv, stream))

ENTRY(qnn_gemm_i8_scaled, 13,
      const char *w = "qnn_gemm_i8_scaled"; int type; real(a[10], &type, w);
      void *x = need(a[0], t_i8, w); int64_t lda = i64(a[1]); void *sa = need(a[2], t_f32, w); void *wt = need(a[3], t_i8, w);
      int64_t ldb = i64(a[4]); void *sb = need(a[5], t_f32, w); void *bias = need(a[6], t_f32, w);
      int64_t M = i64(a[7]) COMMA N = i64(a[8]) COMMA K = i64(a[9]); void *out = any(a[10]); int64_t ldo = i64(a[11]); void *stream = ptr(a[12]),
      qnn_gemm_i8_scaled(x, lda, sa, wt, ldb, sb, bias, M, N, K, out, type, ldo, stream))

ENTRY(qnn_token_logprobs, 12,
      const char *w = "qnn_token_logprobs"; int type; real(a[0], &type, w);
      void *z = any(a[0]); int64_t T = i64(a[1]) COMMA V = i64(a[2]) COMMA ldl = i64(a[3]); void *ids = need(a[4], t_i64, w);
      void *lp = need(a[5], t_f32, w); void *h = need(a[6], t_f32, w); void *lse = need(a[7], t_f32, w); int topk = i32(a[8]);
      void *tl = need(a[9], t_f32, w); void *ti = need(a[10], t_i64, w); void *stream = ptr(a[11]),
      qnn_token_logprobs(z, type, T, V, ldl, ids, lp, h, lse, topk, tl, ti, stream))

ENTRY(qnn_token_logprobs_backward, 12,
      const char *w = "qnn_token_logprobs_backward"; int type; PyObject *dt = real(a[0], &type, w);
      void *z = any(a[0]); int64_t T = i64(a[1]) COMMA V = i64(a[2]) COMMA ldl = i64(a[3]); void *ids = need(a[4], t_i64, w);
      void *lse = need(a[5], t_f32, w); void *h = need(a[6], t_f32, w); void *gl = need(a[7], t_f32, w); void *gh = need(a[8], t_f32, w);
      void *d = need(a[9], dt, w); int64_t ldd = i64(a[10]); void *stream = ptr(a[11]),
      qnn_token_logprobs_backward(z, type, T, V, ldl, ids, lse, h, gl, gh, d, ldd, stream))

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, "status of the C call of this name"}
static PyMethodDef methods[] = {METHOD(qnn_quantize_rows_i8), METHOD(qnn_rmsnorm_quant_i8), METHOD(qnn_silu_mul_quant_i8),
                                METHOD(qnn_gemm_i8_scaled), METHOD(qnn_token_logprobs), METHOD(qnn_token_logprobs_backward),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qnn_calls", "Argument marshalling of libqnn.so calls.", -1, methods,
                                    NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__qnn_calls(void)
{
    PyObject *torch = PyImport_ImportModule("torch");
    if (torch == NULL) return NULL;
    s_dtype = PyUnicode_InternFromString("dtype");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    t_f32 = PyObject_GetAttrString(torch, "float32");
    t_bf16 = PyObject_GetAttrString(torch, "bfloat16");
    t_f16 = PyObject_GetAttrString(torch, "float16");
    t_i8 = PyObject_GetAttrString(torch, "int8");
    t_i64 = PyObject_GetAttrString(torch, "int64");
    Py_DECREF(torch);
    if (!s_dtype || !s_data_ptr || !t_f32 || !t_bf16 || !t_f16 || !t_i8 || !t_i64) return NULL;
    return PyModule_Create(&module);
}
