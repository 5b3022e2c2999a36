/* Calls of the feed-forward entry points from Python without ctypes: what a short call costs the host is marshalling (17 arguments through ctypes take
 * 2.6 us, a routing of 16 tokens takes the GPU 5), so these go through CPython's vector calls instead.  Same arguments in the same order as include/nm.h; a pointer is
 * a tensor (its data_ptr()), an integer or None.  The entry points' addresses come from the library that the package has loaded. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <stdint.h>

typedef int (*route_fn)(const void *, long, const float *, int32_t *, float *, int, int, int, int, int, int, int, int, int, float, void *);
typedef int (*act_fn)(const void *, long, const void *, const void *, const void *, long, void *, long, int, int, int, int, int, int, int, void *, size_t, void *);
typedef int (*moe_fn)(const void *, long, const int32_t *, const float *, const void *, const void *, const void *, long, void *, long, int, int, int, int, int, int,
                      int, int, int, int, void *, size_t, void *);
static route_fn g_route;
static act_fn g_act;
static moe_fn g_moe;
static PyObject *g_data_ptr;                     /* "data_ptr" */

/* The first error stands: what is behind it is not looked at (nothing of Python may be called with an error set), and the caller asks once, after all of the
 * arguments. */
static void *ptr(PyObject *o)
{
    if (o == Py_None || PyErr_Occurred()) return NULL;
    if (PyLong_Check(o)) return PyLong_AsVoidPtr(o);
    PyObject *p = PyObject_CallMethodNoArgs(o, g_data_ptr);
    if (!p) return NULL;
    void *v = PyLong_AsVoidPtr(p);
    Py_DECREF(p);
    return v;
}
static long whole(PyObject *o) { return PyErr_Occurred() ? 0 : PyLong_AsLong(o); }
static int word(PyObject *o)
{
    const long v = whole(o);
    if (v != (int)v && !PyErr_Occurred()) PyErr_SetString(PyExc_OverflowError, "argument does not fit an int");
    return (int)v;
}
static int count_is(Py_ssize_t n, Py_ssize_t want, void *fn)
{
    if (!fn) PyErr_SetString(PyExc_RuntimeError, "no library bound");
    else if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
    else return 1;
    return 0;
}

static PyObject *bind(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "three addresses"); return NULL; }
    void *route = ptr(a[0]), *act = ptr(a[1]), *moe = ptr(a[2]);
    if (PyErr_Occurred()) return NULL;
    g_route = (route_fn)route; g_act = (act_fn)act; g_moe = (moe_fn)moe;
    Py_RETURN_NONE;
}

static PyObject *route(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (!count_is(n, 16, (void *)g_route)) return NULL;
    void *logits = ptr(a[0]), *bias = ptr(a[2]), *experts = ptr(a[3]), *weights = ptr(a[4]), *stream = ptr(a[15]);
    const long ld = whole(a[1]);
    int w[9];
    for (int i = 0; i < 9; ++i) w[i] = word(a[5 + i]);
    const double scale = PyErr_Occurred() ? 0 : PyFloat_AsDouble(a[14]);
    if (PyErr_Occurred()) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_route(logits, ld, (const float *)bias, (int32_t *)experts, (float *)weights, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7], w[8], (float)scale, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

static PyObject *act(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (!count_is(n, 18, (void *)g_act)) return NULL;
    void *A = ptr(a[0]), *B = ptr(a[2]), *bias = ptr(a[3]), *residual = ptr(a[4]), *C = ptr(a[6]), *ws = ptr(a[15]), *stream = ptr(a[17]);
    const long lda = whole(a[1]), ldr = whole(a[5]), ldc = whole(a[7]), bytes = whole(a[16]);
    int w[7];
    for (int i = 0; i < 7; ++i) w[i] = word(a[8 + i]);
    if (PyErr_Occurred()) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_act(A, lda, B, bias, residual, ldr, C, ldc, w[0], w[1], w[2], w[3], w[4], w[5], w[6], ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

static PyObject *moe(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (!count_is(n, 23, (void *)g_moe)) return NULL;
    void *x = ptr(a[0]), *experts = ptr(a[2]), *weights = ptr(a[3]), *up = ptr(a[4]), *down = ptr(a[5]), *residual = ptr(a[6]), *out = ptr(a[8]), *ws = ptr(a[20]),
         *stream = ptr(a[22]);
    const long ldx = whole(a[1]), ldr = whole(a[7]), ldo = whole(a[9]), bytes = whole(a[21]);
    int w[10];
    for (int i = 0; i < 10; ++i) w[i] = word(a[10 + i]);
    if (PyErr_Occurred()) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_moe(x, ldx, (const int32_t *)experts, (const float *)weights, up, down, residual, ldr, out, ldo, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7], w[8], w[9], ws,
                   (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "Addresses of nm_moe_route, nm_matmul_act and nm_moe_ffn."},
    {"nm_moe_route", (PyCFunction)(void (*)(void))route, METH_FASTCALL, "The entry point's arguments; returns its status."},
    {"nm_matmul_act", (PyCFunction)(void (*)(void))act, METH_FASTCALL, "The entry point's arguments; returns its status."},
    {"nm_moe_ffn", (PyCFunction)(void (*)(void))moe, METH_FASTCALL, "The entry point's arguments; returns its status."},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_nm_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__nm_calls(void)
{
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    return g_data_ptr ? PyModule_Create(&module) : NULL;
}
