/*
 * The executor calls of the Python binding, and those of the operators around the products, as C functions.  A small product takes little longer
 * on the GPU than its launch does on the host, and marshalling four arguments through ctypes is a
 * seventh of that: sp.spmm on a 1024 x 512 x 49 layer keeps the host for 2.95 us through ctypes and
 * for 2.55 us through here, and takes 3.15 and 2.65 to 2.85 us per call back to back.
 *
 * Arguments that are not plain integers (or None) go to the ctypes functions handed over by
 * bind(), which accept everything ctypes does; so does the raising of errors.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*execute_fn)(const void *, const void *, void *, void *);

static execute_fn g_run[2];
static PyObject *g_general[2], *g_check, *g_handle;

/* The operators: a descriptor's handle and addresses or sizes, all of them words of the register size. */
enum { RMS_NORM, DEQUANTIZE, ADAPTERS, OPERATORS, MOST_WORDS = 13 };
typedef int (*norm_fn)(const void *, const void *, const void *, const void *, void *, void *, void *, void *, size_t, void *);
typedef int (*dequantize_fn)(const void *, const void *, const void *, const void *, void *, void *);
typedef int (*adapters_fn)(const void *, const void *, const void *, const void *, const void *, const void *, const void *, const void *,
                           const void *, void *, void *, size_t, void *);
static void *g_operator[OPERATORS];
static PyObject *g_operator_general[OPERATORS];
static const Py_ssize_t g_words[OPERATORS] = {10, 6, MOST_WORDS};   /* the last of them is the stream, which may be left out */

/* 1: *out is the address an int or None stands for; 0: something else */
static int address(PyObject *o, void **out) {
    if (o == Py_None) { *out = NULL; return 1; }
    if (!PyLong_CheckExact(o)) return 0;
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) { PyErr_Clear(); return 0; }
    *out = (void *)(uintptr_t)v;
    return 1;
}

static PyObject *execute(int which, PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
    (void)self;
    if (g_check == NULL) {
        PyErr_SetString(PyExc_RuntimeError, "bind() has not been called: import the sparsert module");
        return NULL;
    }
    if (kwnames == NULL && (nargs == 3 || nargs == 4)) {
        PyObject *handle = PyObject_GetAttr(args[0], g_handle);
        if (handle == NULL) return NULL;
        void *p[4] = {NULL, NULL, NULL, NULL};
        const int plain = address(handle, &p[0]) && address(args[1], &p[1]) && address(args[2], &p[2]) && (nargs < 4 || address(args[3], &p[3]));
        Py_DECREF(handle);
        if (plain) {
            int rc;
            Py_BEGIN_ALLOW_THREADS   /* as ctypes does: the runtime may wait for room in its queue */
            rc = g_run[which](p[0], p[1], p[2], p[3]);
            Py_END_ALLOW_THREADS
            if (rc == 0) Py_RETURN_NONE;
            return PyObject_CallFunction(g_check, "i", rc);
        }
    }
    return PyObject_Vectorcall(g_general[which], args, (size_t)nargs, kwnames);
}

static PyObject *spmm(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) { return execute(0, self, args, nargs, kwnames); }
static PyObject *conv3x3(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) { return execute(1, self, args, nargs, kwnames); }

static PyObject *operate(int which, PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
    (void)self;
    if (g_check == NULL || g_operator[which] == NULL) {
        PyErr_SetString(PyExc_RuntimeError, "bind() has not been called: import the sparsert module");
        return NULL;
    }
    if (kwnames == NULL && (nargs == g_words[which] || nargs == g_words[which] - 1)) {
        PyObject *handle = PyObject_GetAttr(args[0], g_handle);
        if (handle == NULL) return NULL;
        void *p[MOST_WORDS] = {NULL};
        int plain = address(handle, &p[0]);
        Py_DECREF(handle);
        for (Py_ssize_t i = 1; plain && i < nargs; ++i) plain = address(args[i], &p[i]);
        if (plain) {
            int rc;
            Py_BEGIN_ALLOW_THREADS
            if (which == RMS_NORM) rc = ((norm_fn)(uintptr_t)g_operator[which])(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], (size_t)(uintptr_t)p[8], p[9]);
            else if (which == DEQUANTIZE) rc = ((dequantize_fn)(uintptr_t)g_operator[which])(p[0], p[1], p[2], p[3], p[4], p[5]);
            else rc = ((adapters_fn)(uintptr_t)g_operator[which])(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], (size_t)(uintptr_t)p[11], p[12]);
            Py_END_ALLOW_THREADS
            if (rc == 0) Py_RETURN_NONE;
            return PyObject_CallFunction(g_check, "i", rc);
        }
    }
    return PyObject_Vectorcall(g_operator_general[which], args, (size_t)nargs, kwnames);
}

static PyObject *rms_norm(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) { return operate(RMS_NORM, self, args, nargs, kwnames); }
static PyObject *dequantize(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) { return operate(DEQUANTIZE, self, args, nargs, kwnames); }
static PyObject *adapters(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) { return operate(ADAPTERS, self, args, nargs, kwnames); }

/* bind_operators(addresses, general functions): three of each, in the order of the enumeration. */
static PyObject *bind_operators(PyObject *self, PyObject *args) {
    unsigned long long at[OPERATORS];
    PyObject *general[OPERATORS];
    (void)self;
    if (!PyArg_ParseTuple(args, "(KKK)(OOO)", &at[0], &at[1], &at[2], &general[0], &general[1], &general[2])) return NULL;
    for (int i = 0; i < OPERATORS; ++i) {
        g_operator[i] = (void *)(uintptr_t)at[i];
        Py_INCREF(general[i]);
        Py_XSETREF(g_operator_general[i], general[i]);
    }
    Py_RETURN_NONE;
}

static PyObject *bind(PyObject *self, PyObject *args) {
    unsigned long long spmm_at, conv_at;
    PyObject *general_spmm, *general_conv, *check;
    (void)self;
    if (!PyArg_ParseTuple(args, "KKOOO", &spmm_at, &conv_at, &general_spmm, &general_conv, &check)) return NULL;
    g_run[0] = (execute_fn)(uintptr_t)spmm_at;
    g_run[1] = (execute_fn)(uintptr_t)conv_at;
    Py_INCREF(general_spmm); Py_INCREF(general_conv); Py_INCREF(check);
    Py_XSETREF(g_general[0], general_spmm);
    Py_XSETREF(g_general[1], general_conv);
    Py_XSETREF(g_check, check);
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"spmm", (PyCFunction)(void (*)(void))spmm, METH_FASTCALL | METH_KEYWORDS,
     "spmm(plan, B_dev, C_dev, stream=0)\n--\n\nsparsert_spmm: device addresses and a hipStream_t as integers."},
    {"conv3x3", (PyCFunction)(void (*)(void))conv3x3, METH_FASTCALL | METH_KEYWORDS,
     "conv3x3(plan, X_dev, Y_dev, stream=0)\n--\n\nsparsert_conv3x3: device addresses and a hipStream_t as integers."},
    {"rms_norm", (PyCFunction)(void (*)(void))rms_norm, METH_FASTCALL | METH_KEYWORDS,
     "rms_norm(norm, X_dev, R_dev, gamma_dev, H_dev, Y_dev, scale_dev=0, workspace_dev=0, workspace_bytes=0, stream=0)\n--\n\n"
     "sparsert_rms_norm: Y = norm(X + R) * gamma, H = X + R; R, gamma, H and the workspace may be 0 (none); scale for an int8 Y only."},
    {"dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL | METH_KEYWORDS,
     "dequantize(dequant, C_dev, row_scale_dev, col_scale_dev, Y_dev, stream=0)\n--\n\nsparsert_dequantize: Y = C * col_scale * row_scale; either scale may be 0 (ones)."},
    {"adapters", (PyCFunction)(void (*)(void))adapters, METH_FASTCALL | METH_KEYWORDS,
     "adapters(adapter_set, X_dev, down_dev, up_dev, index_dev, alpha_dev, C_dev, row_scale_dev, col_scale_dev, Y_dev, workspace_dev, workspace_bytes, stream=0)\n--\n\n"
     "sparsert_adapters: Y = C + alpha up (down x) of every token's adapter; alpha and, for int8 X, the scales may be 0 (ones)."},
    {"bind_operators", bind_operators, METH_VARARGS, "bind_operators(addresses, general functions): set up by the binding."},
    {"bind", bind, METH_VARARGS, "bind(spmm address, conv3x3 address, general spmm, general conv3x3, check): set up by the binding."},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcall(void) {
    g_handle = PyUnicode_InternFromString("handle");
    return g_handle ? PyModule_Create(&module) : NULL;
}
