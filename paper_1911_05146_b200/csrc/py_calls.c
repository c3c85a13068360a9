/* The calls of the linear layer, of label log-probabilities and of distillation from Python: argument marshalling only.
 *
 * A call on a small batch takes the GPU 2 to 3 us; marshalled by ctypes and checked tensor by tensor in Python it took the host 8.  Here
 * the tensors' checks (type, device) and addresses and the current stream are fetched in C and the library's function is called
 * through its address, which setup() gets: this module links neither with the library nor with torch. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "../../include/hpf.h"

static PyObject *g_error;                 /* (status, text) -> raises the package's error */
static PyObject *g_get_device, *g_get_stream;
static PyObject *g_types[3];              /* torch's fp32, bf16, fp16, in the order of hpf_dtype */
static PyObject *g_int32, *g_uint8;
static PyObject *s_dtype, *s_get_device, *s_data_ptr, *s_numel, *s_cuda_stream;

static int (*f_linear_fwd)(const void *, const void *, const void *, const void *, void *, void *, int64_t, int32_t, int32_t, int64_t, int64_t, int32_t, int32_t,
                           void *, size_t, void *);
static int (*f_linear_bwd)(const void *, const void *, const void *, const void *, void *, void *, void *, int64_t, int32_t, int32_t, int64_t, int64_t, int32_t,
                           int32_t, int32_t, void *, size_t, void *);
static int (*f_logprobs_fwd)(const void *, const int32_t *, float *, float *, float *, int32_t *, float *, int64_t, int32_t, int64_t, int32_t, float, int32_t, void *);
static int (*f_logprobs_bwd)(const void *, const int32_t *, const float *, const float *, const float *, const float *, void *, int64_t, int32_t, int64_t, int64_t,
                             float, int32_t, void *);
static int (*f_distill_fwd)(const void *, const int32_t *, const int32_t *, const float *, float *, float *, int64_t, int32_t, int64_t, int32_t, float, float, int32_t,
                            void *);
static int (*f_distill_bwd)(const void *, const int32_t *, const int32_t *, const float *, const float *, const float *, void *, int64_t, int32_t, int64_t, int64_t,
                            int32_t, float, float, int32_t, void *);
static int (*f_distill_fwd_bwd)(const void *, const int32_t *, const int32_t *, const float *, const float *, float *, void *, int64_t, int32_t, int64_t, int64_t,
                                int32_t, float, float, int32_t, void *);

/* A failed check: raises the package's error through g_error.  Always 0. */
static int refuse(int status, const char *what, PyObject *t)
{
    PyObject *r = PyObject_CallFunction(g_error, "isO", status, what, t);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, what);
    return 0;
}

typedef struct {
    long device;
    int dtype;                             /* of the call: HPF_FP32, HPF_BF16 or HPF_FP16 */
} Call;

static long method_long(PyObject *t, PyObject *name)
{
    PyObject *r = PyObject_CallMethodNoArgs(t, name);
    if (!r) return -1;
    const long v = PyLong_AsLong(r);
    Py_DECREF(r);
    return v;
}

/* The address of a tensor of the wanted type on the call's device; NULL for None.  0 = refused. */
static int address(const Call *c, PyObject *t, PyObject *type, const char *name, void *out)
{
    *(void **)out = NULL;
    if (t == Py_None) return 1;
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return 0;
    const int same = d == type;
    Py_DECREF(d);
    if (!same) return refuse(HPF_ERR_INVALID, name, t);
    if (method_long(t, s_get_device) != c->device) return PyErr_Occurred() ? 0 : refuse(HPF_ERR_INVALID, name, t);
    PyObject *p = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!p) return 0;
    *(void **)out = PyLong_AsVoidPtr(p);
    Py_DECREF(p);
    return !PyErr_Occurred();
}
/* Which of the three types a tensor has; -1 = refused. */
static int type_of(PyObject *t, const char *name)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    Py_DECREF(d);                          /* torch keeps its dtypes */
    for (int i = 0; i < 3; ++i)
        if (d == g_types[i]) return i;
    refuse(HPF_ERR_INVALID, name, t);
    return -1;
}
static int begin(Call *c, PyObject *first, const char *name)
{
    PyObject *d = PyObject_CallNoArgs(g_get_device);
    if (!d) return 0;
    c->device = PyLong_AsLong(d);
    Py_DECREF(d);
    c->dtype = type_of(first, name);
    return c->dtype >= 0 && !PyErr_Occurred();
}
static int stream_of(const Call *c, PyObject *s, void **out)
{
    PyObject *h;
    if (s == Py_None) h = PyObject_CallFunction(g_get_stream, "l", c->device);
    else if (PyLong_Check(s)) h = Py_NewRef(s);
    else h = PyObject_GetAttr(s, s_cuda_stream);
    if (!h) return 0;
    *out = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}
static int i64(PyObject *o, int64_t *v) { *v = PyLong_AsLongLong(o); return !PyErr_Occurred(); }
static int i32(PyObject *o, int32_t *v)
{
    const long long w = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) return 0;
    if (w != (int32_t)w) { PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits"); return 0; }
    *v = (int32_t)w;
    return 1;
}
static int f32(PyObject *o, float *v) { *v = (float)PyFloat_AsDouble(o); return !PyErr_Occurred(); }

static PyObject *done(int status)
{
    if (status != HPF_OK) {
        refuse(status, "", Py_None);
        return NULL;
    }
    Py_RETURN_NONE;
}
#define ARGS(n) \
    if (nargs != n) { PyErr_Format(PyExc_TypeError, "%d arguments are wanted, got %zd", n, nargs); return NULL; }
#define LAUNCH(call) \
    int status; \
    Py_BEGIN_ALLOW_THREADS status = call; \
    Py_END_ALLOW_THREADS return done(status)

static PyObject *linear_fwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    ARGS(14)
    Call c;
    void *x, *w, *bias, *residual, *y, *z, *scratch, *st;
    int64_t rows, ld_x, ld_y;
    int32_t n_in, n_out, act;
    if (!begin(&c, a[0], "x")) return NULL;
    PyObject *t = g_types[c.dtype];
    if (!address(&c, a[0], t, "x", &x) || !address(&c, a[1], t, "w", &w) || !address(&c, a[2], t, "bias", &bias) || !address(&c, a[3], t, "residual", &residual) ||
        !address(&c, a[4], t, "y", &y) || !address(&c, a[5], t, "z", &z) || !i64(a[6], &rows) || !i32(a[7], &n_in) || !i32(a[8], &n_out) || !i64(a[9], &ld_x) ||
        !i64(a[10], &ld_y) || !i32(a[11], &act) || !address(&c, a[12], g_uint8, "scratch", &scratch) || !stream_of(&c, a[13], &st))
        return NULL;
    const long bytes = a[12] == Py_None ? 0 : method_long(a[12], s_numel);
    if (PyErr_Occurred()) return NULL;
    LAUNCH(f_linear_fwd(x, w, bias, residual, y, z, rows, n_in, n_out, ld_x, ld_y, c.dtype, act, scratch, (size_t)bytes, st));
}

static PyObject *linear_bwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    ARGS(15)
    Call c;
    void *dy, *z, *x, *w, *dx, *dw, *db, *scratch, *st;
    int64_t rows, ld_x, ld_y;
    int32_t n_in, n_out, act;
    if (!begin(&c, a[0], "dy")) return NULL;
    PyObject *t = g_types[c.dtype];
    int grad = c.dtype;                    /* the gradients of the weights may be fp32 whatever the rest is */
    if (a[5] != Py_None) grad = type_of(a[5], "dw");
    else if (a[6] != Py_None) grad = type_of(a[6], "dbias");
    if (grad < 0) return NULL;
    PyObject *g = g_types[grad];
    if (!address(&c, a[0], t, "dy", &dy) || !address(&c, a[1], t, "z", &z) || !address(&c, a[2], t, "x", &x) || !address(&c, a[3], t, "w", &w) ||
        !address(&c, a[4], t, "dx", &dx) || !address(&c, a[5], g, "dw", &dw) || !address(&c, a[6], g, "dbias", &db) || !i64(a[7], &rows) || !i32(a[8], &n_in) ||
        !i32(a[9], &n_out) || !i64(a[10], &ld_x) || !i64(a[11], &ld_y) || !i32(a[12], &act) || !address(&c, a[13], g_uint8, "scratch", &scratch) ||
        !stream_of(&c, a[14], &st))
        return NULL;
    const long bytes = a[13] == Py_None ? 0 : method_long(a[13], s_numel);
    if (PyErr_Occurred()) return NULL;
    LAUNCH(f_linear_bwd(dy, z, x, w, dx, dw, db, rows, n_in, n_out, ld_x, ld_y, c.dtype, act, grad, scratch, (size_t)bytes, st));
}

static PyObject *logprobs_fwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    ARGS(13)
    Call c;
    void *logits, *labels, *lp, *h, *lse, *ids, *top, *st;
    int64_t rows, ld;
    int32_t classes, k;
    float temperature;
    PyObject *f = g_types[HPF_FP32];
    if (!begin(&c, a[0], "logits") || !address(&c, a[0], g_types[c.dtype], "logits", &logits) || !address(&c, a[1], g_int32, "labels", &labels) ||
        !address(&c, a[2], f, "logprob", &lp) || !address(&c, a[3], f, "entropy", &h) || !address(&c, a[4], f, "lse", &lse) ||
        !address(&c, a[5], g_int32, "top_ids", &ids) || !address(&c, a[6], f, "top_logprobs", &top) || !i64(a[7], &rows) || !i32(a[8], &classes) || !i64(a[9], &ld) ||
        !i32(a[10], &k) || !f32(a[11], &temperature) || !stream_of(&c, a[12], &st))
        return NULL;
    LAUNCH(f_logprobs_fwd(logits, labels, lp, h, lse, ids, top, rows, classes, ld, k, temperature, c.dtype, st));
}

static PyObject *logprobs_bwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    ARGS(13)
    Call c;
    void *logits, *labels, *lse, *h, *g, *e, *out, *st;
    int64_t rows, ld, ld_d;
    int32_t classes;
    float temperature;
    PyObject *f = g_types[HPF_FP32];
    if (!begin(&c, a[0], "logits") || !address(&c, a[0], g_types[c.dtype], "logits", &logits) || !address(&c, a[1], g_int32, "labels", &labels) ||
        !address(&c, a[2], f, "lse", &lse) || !address(&c, a[3], f, "entropy", &h) || !address(&c, a[4], f, "d_logprob", &g) ||
        !address(&c, a[5], f, "d_entropy", &e) || !address(&c, a[6], g_types[c.dtype], "d_logits", &out) || !i64(a[7], &rows) || !i32(a[8], &classes) ||
        !i64(a[9], &ld) || !i64(a[10], &ld_d) || !f32(a[11], &temperature) || !stream_of(&c, a[12], &st))
        return NULL;
    LAUNCH(f_logprobs_bwd(logits, labels, lse, h, g, e, out, rows, classes, ld, ld_d, temperature, c.dtype, st));
}

static PyObject *distill_fwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    ARGS(13)
    Call c;
    void *logits, *labels, *ids, *teacher, *loss, *stats, *st;
    int64_t rows, ld;
    int32_t classes, k;
    float temperature, alpha;
    PyObject *f = g_types[HPF_FP32];
    if (!begin(&c, a[0], "logits") || !address(&c, a[0], g_types[c.dtype], "logits", &logits) || !address(&c, a[1], g_int32, "labels", &labels) ||
        !address(&c, a[2], g_int32, "teacher_ids", &ids) || !address(&c, a[3], f, "teacher_logits", &teacher) || !address(&c, a[4], f, "loss", &loss) ||
        !address(&c, a[5], f, "stats", &stats) || !i64(a[6], &rows) || !i32(a[7], &classes) || !i64(a[8], &ld) || !i32(a[9], &k) || !f32(a[10], &temperature) ||
        !f32(a[11], &alpha) || !stream_of(&c, a[12], &st))
        return NULL;
    LAUNCH(f_distill_fwd(logits, labels, ids, teacher, loss, stats, rows, classes, ld, k, temperature, alpha, c.dtype, st));
}

/* distill_bwd (stats, d_loss, d_logits) and distill_fwd_bwd (d_loss, loss, d_logits) take the same arguments but for two names */
static PyObject *distill_grad(PyObject *const *a, Py_ssize_t nargs, int both)
{
    ARGS(15)
    Call c;
    void *logits, *labels, *ids, *teacher, *p, *q, *out, *st;
    int64_t rows, ld, ld_d;
    int32_t classes, k;
    float temperature, alpha;
    PyObject *f = g_types[HPF_FP32];
    if (!begin(&c, a[0], "logits") || !address(&c, a[0], g_types[c.dtype], "logits", &logits) || !address(&c, a[1], g_int32, "labels", &labels) ||
        !address(&c, a[2], g_int32, "teacher_ids", &ids) || !address(&c, a[3], f, "teacher_logits", &teacher) || !address(&c, a[4], f, both ? "d_loss" : "stats", &p) ||
        !address(&c, a[5], f, both ? "loss" : "d_loss", &q) || !address(&c, a[6], g_types[c.dtype], "d_logits", &out) || !i64(a[7], &rows) || !i32(a[8], &classes) ||
        !i64(a[9], &ld) || !i64(a[10], &ld_d) || !i32(a[11], &k) || !f32(a[12], &temperature) || !f32(a[13], &alpha) || !stream_of(&c, a[14], &st))
        return NULL;
    if (both) {
        LAUNCH(f_distill_fwd_bwd(logits, labels, ids, teacher, p, q, out, rows, classes, ld, ld_d, k, temperature, alpha, c.dtype, st));
    }
    LAUNCH(f_distill_bwd(logits, labels, ids, teacher, p, q, out, rows, classes, ld, ld_d, k, temperature, alpha, c.dtype, st));
}
static PyObject *distill_bwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs) { return distill_grad(a, nargs, 0); }
static PyObject *distill_fwd_bwd(PyObject *self, PyObject *const *a, Py_ssize_t nargs) { return distill_grad(a, nargs, 1); }

/* setup(error, get_device, get_stream, (fp32, bf16, fp16, int32, uint8), (addresses in the order below)) */
static PyObject *setup(PyObject *self, PyObject *args)
{
    PyObject *types[5];
    unsigned long long f[7];
    if (!PyArg_ParseTuple(args, "OOO(OOOOO)(KKKKKKK)", &g_error, &g_get_device, &g_get_stream, &types[0], &types[1], &types[2], &types[3], &types[4], &f[0], &f[1],
                          &f[2], &f[3], &f[4], &f[5], &f[6]))
        return NULL;
    for (int i = 0; i < 3; ++i) g_types[i] = Py_NewRef(types[i]);
    g_int32 = Py_NewRef(types[3]);
    g_uint8 = Py_NewRef(types[4]);
    Py_INCREF(g_error);
    Py_INCREF(g_get_device);
    Py_INCREF(g_get_stream);
    void *const to[7] = {&f_linear_fwd, &f_linear_bwd, &f_logprobs_fwd, &f_logprobs_bwd, &f_distill_fwd, &f_distill_bwd, &f_distill_fwd_bwd};
    for (int i = 0; i < 7; ++i) {
        const uintptr_t at = (uintptr_t)f[i];
        memcpy(to[i], &at, sizeof at);
    }
    Py_RETURN_NONE;
}

#define CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, NULL}, CALL(linear_fwd), CALL(linear_bwd), CALL(logprobs_fwd), CALL(logprobs_bwd),
                                CALL(distill_fwd), CALL(distill_bwd), CALL(distill_fwd_bwd), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void)
{
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return PyModule_Create(&module);
}
