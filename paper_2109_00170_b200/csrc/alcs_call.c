// The calls that a program makes once per layer, marshalled in C: the same functions of libalcs.so that binding.py
// declares through ctypes, which spends about 2 us per call on a dozen arguments, a quarter of a small layer's pass.
// The addresses of the functions come from the library that binding.py has loaded (bind), so there is one library
// and one set of entry points.  Only the plain forms of arguments are taken here: Python integers, None, what has a
// data_ptr() or a cuda_stream that is such an integer.  For any other call (numpy integers, arrays, ctypes objects, what is
// wrong) the answer is None and nothing has been called: binding.py then makes it through ctypes, whose conversions
// and errors are the interface.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

typedef int (*spconv1x1_fn)(const void*, const void*, void*, int, int, int, const float*, unsigned, void*);
typedef int (*spconv1x1_ex_fn)(const void*, const void*, void*, int, int, int, int, const float*, const void*, unsigned, const void*, void*);
typedef int (*spconv2d_fn)(const void*, const void*, void*, int, int, int, int, int, int, int, int, const float*, unsigned, void*);
typedef int (*stack_run_fn)(void*, void*);

typedef int (*group_norm_fn)(const void*, void*, int, int, int, int, int, const float*, const float*, float, unsigned, int, float*, float*, void*, size_t, void*);
typedef int (*group_norm_backward_fn)(const void*, const void*, void*, int, int, int, int, int, const float*, const float*, const float*, const float*, float*,
                                      float*, unsigned, int, void*, size_t, void*);
typedef int (*mx4_quantize_fn)(const void*, int, int, long long, int, void*, void*, void*);
typedef int (*mx4_dequantize_fn)(const void*, const void*, int, int, void*, long long, int, void*);
typedef int (*mx4_product_fn)(const void*, const void*, int, const void*, const void*, int, int, void*, const float*, const void*, unsigned, int, void*);

static group_norm_fn f_group_norm;
static group_norm_backward_fn f_group_norm_backward;
static mx4_quantize_fn f_mx4_quantize;
static mx4_dequantize_fn f_mx4_dequantize;
static mx4_product_fn f_mx4_product;
static spconv1x1_fn f_spconv1x1;
static spconv1x1_ex_fn f_spconv1x1_ex;
static spconv2d_fn f_spconv2d;
static stack_run_fn f_stack_run;
static PyObject *s_data_ptr, *s_cuda_stream, *s_value;

// An address of a Python integer that fits one.
static int to_ptr(PyObject* o, void** out)
{
    if (!PyLong_Check(o)) return 0;
    *out = PyLong_AsVoidPtr(o);
    return *out || !PyErr_Occurred();
}

// Of a ctypes.c_void_p that is not null.
static int handle(PyObject* o, void** out)
{
    PyObject* v = PyObject_GetAttr(o, s_value);
    const int ok = v && to_ptr(v, out) && *out;
    Py_XDECREF(v);
    return ok;
}

static int address(PyObject* o, void** out)
{
    if (o == Py_None) { *out = NULL; return 1; }
    if (PyLong_Check(o)) return to_ptr(o, out);
    PyObject* v = PyObject_CallMethodNoArgs(o, s_data_ptr);
    const int ok = v && to_ptr(v, out);
    Py_XDECREF(v);
    return ok;
}

static int stream_of(PyObject* o, void** out)
{
    if (o == Py_None) { *out = NULL; return 1; }
    if (PyLong_Check(o)) return to_ptr(o, out);
    PyObject* v = PyObject_GetAttr(o, s_cuda_stream);
    const int ok = v && (v == Py_None ? (*out = NULL, 1) : to_ptr(v, out));
    Py_XDECREF(v);
    return ok;
}

// C's int of a Python integer: the low bits, as ctypes takes them.
static int integer(PyObject* o, int* out)
{
    if (!PyLong_Check(o)) return 0;
    const unsigned long v = PyLong_AsUnsignedLongMask(o);
    if (v == (unsigned long)-1 && PyErr_Occurred()) return 0;
    *out = (int)v;
    return 1;
}

// Not a plain call: None, and whatever was raised on the way is raised again where ctypes meets it.
static PyObject* not_plain(void)
{
    if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return NULL;      // (an interrupt)
    PyErr_Clear();
    Py_RETURN_NONE;
}

static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void* f[4];
    (void)self;
    for (int i = 0; i < 4; ++i)
        if (n != 4 || !to_ptr(a[i], &f[i])) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "four addresses expected");
            return NULL;
        }
    f_spconv1x1 = (spconv1x1_fn)f[0];
    f_spconv1x1_ex = (spconv1x1_ex_fn)f[1];
    f_spconv2d = (spconv2d_fn)f[2];
    f_stack_run = (stack_run_fn)f[3];
    Py_RETURN_NONE;
}

// Each: the status, or None.  w, x, y, n, h, wd, bias, flags, stream
static PyObject* spconv1x1(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void *w, *x, *y, *bias, *st;
    int d[3], flags, rc;
    (void)self;
    if (n != 9 || !handle(a[0], &w) || !address(a[1], &x) || !address(a[2], &y)) return not_plain();
    for (int i = 0; i < 3; ++i)
        if (!integer(a[3 + i], &d[i])) return not_plain();
    if (!address(a[6], &bias) || !integer(a[7], &flags) || !stream_of(a[8], &st)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_spconv1x1(w, x, y, d[0], d[1], d[2], bias, (unsigned)flags, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// w, x, y, n, h, wd, stride, bias, residual, flags, stream
static PyObject* spconv1x1_ex(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void *w, *x, *y, *bias, *res, *st;
    int d[4], flags, rc;
    (void)self;
    if (n != 11 || !handle(a[0], &w) || !address(a[1], &x) || !address(a[2], &y)) return not_plain();
    for (int i = 0; i < 4; ++i)
        if (!integer(a[3 + i], &d[i])) return not_plain();
    if (!address(a[7], &bias) || !address(a[8], &res) || !integer(a[9], &flags) || !stream_of(a[10], &st)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_spconv1x1_ex(w, x, y, d[0], d[1], d[2], d[3], bias, res, (unsigned)flags, NULL, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// w, x, y, n, cin, h, wd, kh, kw, stride, pad, bias, flags, stream
static PyObject* spconv2d(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void *w, *x, *y, *bias, *st;
    int d[8], flags, rc;
    (void)self;
    if (n != 14 || !handle(a[0], &w) || !address(a[1], &x) || !address(a[2], &y)) return not_plain();
    for (int i = 0; i < 8; ++i)
        if (!integer(a[3 + i], &d[i])) return not_plain();
    if (!address(a[11], &bias) || !integer(a[12], &flags) || !stream_of(a[13], &st)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_spconv2d(w, x, y, d[0], d[1], d[2], d[3], d[4], d[5], d[6], d[7], bias, (unsigned)flags, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// stack, stream
static PyObject* stack_run(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void *s, *st;
    int rc;
    (void)self;
    if (n != 2 || !handle(a[0], &s) || !stream_of(a[1], &st)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_stack_run(s, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* bind_dense(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void* f[5];
    (void)self;
    for (int i = 0; i < 5; ++i)
        if (n != 5 || !to_ptr(a[i], &f[i])) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "five addresses expected");
            return NULL;
        }
    f_group_norm = (group_norm_fn)f[0];
    f_group_norm_backward = (group_norm_backward_fn)f[1];
    f_mx4_quantize = (mx4_quantize_fn)f[2];
    f_mx4_dequantize = (mx4_dequantize_fn)f[3];
    f_mx4_product = (mx4_product_fn)f[4];
    Py_RETURN_NONE;
}

// An argument of the calls below, by the letter of its kind: p address, i int, l 64 bits (long long, size_t), f float, s stream.
typedef union { void* p; int i; unsigned long long l; float f; } value;

static int take(const char* kinds, PyObject* const* a, Py_ssize_t n, value* v)
{
    Py_ssize_t k = 0;
    for (; kinds[k]; ++k) {
        if (k >= n) return 0;
        switch (kinds[k]) {
        case 'p': if (!address(a[k], &v[k].p)) return 0; break;
        case 's': if (!stream_of(a[k], &v[k].p)) return 0; break;
        case 'i': if (!integer(a[k], &v[k].i)) return 0; break;
        case 'f':
            if (!PyFloat_Check(a[k])) return 0;
            v[k].f = (float)PyFloat_AS_DOUBLE(a[k]);
            break;
        default:
            if (!PyLong_Check(a[k])) return 0;
            v[k].l = PyLong_AsUnsignedLongLongMask(a[k]);
            if (v[k].l == (unsigned long long)-1 && PyErr_Occurred()) return 0;
        }
    }
    return k == n;
}

// x, y, n, h, wd, c, groups, gamma, beta, eps, flags, dt, mean, rstd, workspace, bytes, stream
static PyObject* group_norm(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    value v[17];
    int rc;
    (void)self;
    if (!take("ppiiiiippfiipppls", a, n, v)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_group_norm(v[0].p, v[1].p, v[2].i, v[3].i, v[4].i, v[5].i, v[6].i, v[7].p, v[8].p, v[9].f, (unsigned)v[10].i, v[11].i, v[12].p, v[13].p, v[14].p,
                      (size_t)v[15].l, v[16].p);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// x, dy, dx, n, h, wd, c, groups, mean, rstd, gamma, beta, dgamma, dbeta, flags, dt, workspace, bytes, stream
static PyObject* group_norm_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    value v[19];
    int rc;
    (void)self;
    if (!take("pppiiiiippppppiipls", a, n, v)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_group_norm_backward(v[0].p, v[1].p, v[2].p, v[3].i, v[4].i, v[5].i, v[6].i, v[7].i, v[8].p, v[9].p, v[10].p, v[11].p, v[12].p, v[13].p,
                               (unsigned)v[14].i, v[15].i, v[16].p, (size_t)v[17].l, v[18].p);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// x, rows, cols, ldx, dt, data, scales, stream
static PyObject* mx4_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    value v[8];
    int rc;
    (void)self;
    if (!take("piilipps", a, n, v)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_mx4_quantize(v[0].p, v[1].i, v[2].i, (long long)v[3].l, v[4].i, v[5].p, v[6].p, v[7].p);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// data, scales, rows, cols, y, ldy, dt, stream
static PyObject* mx4_dequantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    value v[8];
    int rc;
    (void)self;
    if (!take("ppiiplis", a, n, v)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_mx4_dequantize(v[0].p, v[1].p, v[2].i, v[3].i, v[4].p, (long long)v[5].l, v[6].i, v[7].p);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// x, x_scales, rows, w, w_scales, cout, cin, y, bias, residual, flags, dt, stream
static PyObject* mx4_product(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    value v[13];
    int rc;
    (void)self;
    if (!take("ppippiipppiis", a, n, v)) return not_plain();
    Py_BEGIN_ALLOW_THREADS
    rc = f_mx4_product(v[0].p, v[1].p, v[2].i, v[3].p, v[4].p, v[5].i, v[6].i, v[7].p, v[8].p, v[9].p, (unsigned)v[10].i, v[11].i, v[12].p);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, NULL},
                                {"spconv1x1", (PyCFunction)(void (*)(void))spconv1x1, METH_FASTCALL, NULL},
                                {"spconv1x1_ex", (PyCFunction)(void (*)(void))spconv1x1_ex, METH_FASTCALL, NULL},
                                {"spconv2d", (PyCFunction)(void (*)(void))spconv2d, METH_FASTCALL, NULL},
                                {"bind_dense", (PyCFunction)(void (*)(void))bind_dense, METH_FASTCALL, NULL},
                                {"group_norm", (PyCFunction)(void (*)(void))group_norm, METH_FASTCALL, NULL},
                                {"group_norm_backward", (PyCFunction)(void (*)(void))group_norm_backward, METH_FASTCALL, NULL},
                                {"mx4_quantize", (PyCFunction)(void (*)(void))mx4_quantize, METH_FASTCALL, NULL},
                                {"mx4_dequantize", (PyCFunction)(void (*)(void))mx4_dequantize, METH_FASTCALL, NULL},
                                {"mx4_product", (PyCFunction)(void (*)(void))mx4_product, METH_FASTCALL, NULL},
                                {"stack_run", (PyCFunction)(void (*)(void))stack_run, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_alcs_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__alcs_call(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_value = PyUnicode_InternFromString("value");
    if (!s_data_ptr || !s_cuda_stream || !s_value) return NULL;
    return PyModule_Create(&module);
}
