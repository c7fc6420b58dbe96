/* Argument marshalling of the calls a training step makes, as a CPython extension: None is NULL, an int is an address or a number, a tensor is
 * asked for its data_ptr(); at a fifth of the time that ctypes and the helpers in cgbn.py take for the same (a step of a small layer is
 * host bound: of 9 us a call they took 4).  Whatever is not so plain (a ctypes object, a wrong type, a name that is not in the table) is
 * answered NotImplemented before anything is called, and cgbn.py takes the call through ctypes, which accepts or refuses it.  The library is not
 * linked: bind() is handed the addresses of its functions by whoever loaded it. */

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "cgbn.h"

typedef cgbn_status (*forward_fn)(const void*, int, int, int, int, cgbn_layout, int, const float*, const float*, float, void*, float*, float*,
                                  cgbn_dtype, float*, void*, size_t, void*);
typedef cgbn_status (*forward_relu_fn)(const void*, const void*, int, int, int, int, cgbn_layout, int, const float*, const float*, float, void*,
                                       float*, float*, cgbn_dtype, float*, void*, size_t, void*);
typedef cgbn_status (*backward_fn)(const void*, const void*, const float*, const float*, const float*, void*, float*, float*, int, int, int, int,
                                   cgbn_layout, int, cgbn_dtype, const float*, void*, size_t, void*);
typedef cgbn_status (*backward_relu_fn)(const void*, const void*, const void*, const float*, const float*, const float*, void*, void*, float*,
                                        float*, int, int, int, int, cgbn_layout, int, cgbn_dtype, const float*, void*, size_t, void*);
typedef cgbn_status (*frozen_forward_fn)(const void*, int, int, int, int, cgbn_layout, cgbn_dtype, const float*, const float*, const float*,
                                         const float*, float, void*, void*);
typedef cgbn_status (*frozen_backward_fn)(const void*, int, int, int, int, cgbn_layout, cgbn_dtype, const float*, const float*, float, void*,
                                          void*);

typedef cgbn_status (*linear_forward_fn)(const void*, const void*, const float*, const void*, long long, int, int, cgbn_activation, void*, void*,
                                         cgbn_dtype, void*, size_t, void*);
typedef cgbn_status (*linear_backward_fn)(const void*, const void*, const void*, const void*, long long, int, int, cgbn_activation, void*, void*,
                                          float*, void*, cgbn_dtype, void*, size_t, void*);
typedef cgbn_status (*gated_forward_fn)(const void*, const void*, const void*, long long, int, int, cgbn_activation, void*, void*, void*, cgbn_dtype,
                                        void*, size_t, void*);
typedef cgbn_status (*gated_backward_fn)(const void*, const void*, const void*, const void*, const void*, const void*, long long, int, int,
                                         cgbn_activation, void*, void*, void*, cgbn_dtype, void*, size_t, void*);
typedef cgbn_status (*head_norm_forward_fn)(const void*, long long, const void*, long long, long long, int, int, int, int, cgbn_rotation, const int*,
                                            const float*, const float*, int, const float*, const float*, float, void*, long long, void*, long long,
                                            cgbn_dtype, void*);
typedef cgbn_status (*head_norm_backward_fn)(const void*, long long, const void*, long long, const void*, long long, const void*, long long, long long,
                                             int, int, int, int, cgbn_rotation, const int*, const float*, const float*, int, const float*,
                                             const float*, float, void*, long long, void*, long long, float*, float*, cgbn_dtype, void*, size_t, void*);

typedef cgbn_status (*rotate_fn)(const void*, long long, const void*, long long, long long, int, int, int, int, cgbn_rotation, const int*, const double*,
                                 float, void*, long long, void*, long long, cgbn_dtype, void*);
typedef cgbn_status (*page_plan_fn)(const int*, const int*, int, int, const int*, int, const int*, int*, int*, int, int, int, long long, int*, int*, int*,
                                    int*, void*, size_t, void*);
typedef cgbn_status (*page_store_fn)(const void*, long long, const void*, long long, long long, int, int, const int*, void*, void*, int, int, cgbn_dtype,
                                     void*);
typedef cgbn_status (*prefix_attention_fn)(const void*, long long, long long, int, const int*, const int*, int, int, int, float, const void*, const void*,
                                           int, int, const int*, int, const int*, int, void*, long long, float*, cgbn_dtype, void*, size_t, void*);

static rotate_fn g_rotate_forward, g_rotate_backward;
static page_plan_fn g_page_plan;
static page_store_fn g_page_store;
static prefix_attention_fn g_prefix_attention;
static linear_forward_fn g_linear_forward;
static linear_backward_fn g_linear_backward;
static gated_forward_fn g_gated_forward;
static gated_backward_fn g_gated_backward;
static head_norm_forward_fn g_head_norm_forward;
static head_norm_backward_fn g_head_norm_backward;
static PyObject *g_activations, *g_rotations;           /* name -> number */
static forward_fn g_forward;
static forward_relu_fn g_forward_relu;
static backward_fn g_backward;
static backward_relu_fn g_backward_relu;
static frozen_forward_fn g_frozen_forward;
static frozen_backward_fn g_frozen_backward;
static PyObject *g_layouts, *g_dtypes, *g_stream;       /* name -> number; () -> the current stream's address */
static PyObject *g_data_ptr, *g_numel, *g_element_size;

/* Converters: each returns 0 and clears *plain for what ctypes has to deal with, and does nothing once *plain is 0. */
static unsigned long long number(PyObject* o, int* plain)
{
    if (*plain && PyLong_Check(o)) return PyLong_AsUnsignedLongLongMask(o);
    *plain = 0;
    return 0;
}
/* the number that a method without arguments returns */
static unsigned long long asked(PyObject* o, PyObject* method, int* plain)
{
    unsigned long long v;
    PyObject* a = PyObject_CallMethodNoArgs(o, method);
    if (!a) { *plain = 0; return 0; }
    v = number(a, plain);
    Py_DECREF(a);
    return v;
}
static void* ptr(PyObject* o, int* plain)
{
    if (!*plain || o == Py_None) return NULL;
    return (void*)(uintptr_t)(PyLong_Check(o) ? number(o, plain) : asked(o, g_data_ptr, plain));
}
static int num(PyObject* o, int* plain)
{
    return (int)number(o, plain);
}
static long long wide(PyObject* o, int* plain)
{
    return (long long)number(o, plain);
}
static int name(PyObject* table, PyObject* o, int* plain)
{
    if (*plain && PyUnicode_Check(o)) {
        o = PyDict_GetItemWithError(table, o);        /* borrowed */
        if (!o) { *plain = 0; return 0; }
    }
    return (int)number(o, plain);
}
static float real(PyObject* o, int* plain)
{
    if (*plain && PyFloat_Check(o)) return (float)PyFloat_AS_DOUBLE(o);
    *plain = 0;
    return 0.f;
}
/* the workspace's size: what the caller says, else the tensor's own */
static size_t room(PyObject* workspace, PyObject* bytes, int* plain)
{
    unsigned long long n;
    if (!*plain) return 0;
    if (bytes != Py_None) return (size_t)number(bytes, plain);
    if (workspace == Py_None) return 0;
    n = asked(workspace, g_numel, plain);
    return *plain ? (size_t)(n * asked(workspace, g_element_size, plain)) : 0;
}
static void* stream(PyObject* o, int* plain)
{
    void* v;
    PyObject* a;
    if (!*plain) return NULL;
    if (PyLong_Check(o)) return (void*)(uintptr_t)number(o, plain);
    a = PyObject_CallOneArg(g_stream, o);
    if (!a) { *plain = 0; return NULL; }
    v = a == Py_None ? NULL : (void*)(uintptr_t)number(a, plain);
    Py_DECREF(a);
    return v;
}

#define ARGS(count_)                                                                                     \
    int plain = 1;                                                                                       \
    if (n != (count_)) { PyErr_Format(PyExc_TypeError, "%d arguments, %zd given", (count_), n); return NULL; } \
    if (!g_forward) { PyErr_SetString(PyExc_RuntimeError, "bind() first"); return NULL; }
/* (the launch may wait for room in a queue) */
#define CALL(call_)                                                                                      \
    do {                                                                                                 \
        cgbn_status s_;                                                                                  \
        if (!plain) {                                                                                    \
            if (PyErr_Occurred()) {                                                                      \
                if (!PyErr_ExceptionMatches(PyExc_Exception)) return NULL;       /* an interrupt */      \
                PyErr_Clear();                                                                           \
            }                                                                                            \
            Py_RETURN_NOTIMPLEMENTED;                                                                    \
        }                                                                                                \
        Py_BEGIN_ALLOW_THREADS                                                                           \
        s_ = (call_);                                                                                    \
        Py_END_ALLOW_THREADS                                                                             \
        return PyLong_FromLong((long)s_);                                                                \
    } while (0)

static PyObject* forward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    ARGS(18)
    const void* x = ptr(a[0], &plain);
    const int N = num(a[1], &plain), C = num(a[2], &plain), H = num(a[3], &plain), W = num(a[4], &plain), layout = name(g_layouts, a[5], &plain), K = num(a[6], &plain);
    const float *gamma = ptr(a[7], &plain), *beta = ptr(a[8], &plain);
    const float eps = real(a[9], &plain);
    void* y = ptr(a[10], &plain);
    float *mean = ptr(a[11], &plain), *invstd = ptr(a[12], &plain);
    const int dtype = name(g_dtypes, a[13], &plain);
    float* mean_lo = ptr(a[14], &plain);
    void* ws = ptr(a[15], &plain);
    const size_t bytes = room(a[15], a[16], &plain);
    void* st = stream(a[17], &plain);
    CALL(g_forward(x, N, C, H, W, layout, K, gamma, beta, eps, y, mean, invstd, dtype, mean_lo, ws, bytes, st));
}
static PyObject* forward_relu(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    ARGS(19)
    const void *x = ptr(a[0], &plain), *shortcut = ptr(a[1], &plain);
    const int N = num(a[2], &plain), C = num(a[3], &plain), H = num(a[4], &plain), W = num(a[5], &plain), layout = name(g_layouts, a[6], &plain), K = num(a[7], &plain);
    const float *gamma = ptr(a[8], &plain), *beta = ptr(a[9], &plain);
    const float eps = real(a[10], &plain);
    void* y = ptr(a[11], &plain);
    float *mean = ptr(a[12], &plain), *invstd = ptr(a[13], &plain);
    const int dtype = name(g_dtypes, a[14], &plain);
    float* mean_lo = ptr(a[15], &plain);
    void* ws = ptr(a[16], &plain);
    const size_t bytes = room(a[16], a[17], &plain);
    void* st = stream(a[18], &plain);
    CALL(g_forward_relu(x, shortcut, N, C, H, W, layout, K, gamma, beta, eps, y, mean, invstd, dtype, mean_lo, ws, bytes, st));
}
static PyObject* backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    ARGS(19)
    const void *dy = ptr(a[0], &plain), *x = ptr(a[1], &plain);
    const float *mean = ptr(a[2], &plain), *invstd = ptr(a[3], &plain), *gamma = ptr(a[4], &plain);
    void* dx = ptr(a[5], &plain);
    float *dgamma = ptr(a[6], &plain), *dbeta = ptr(a[7], &plain);
    const int N = num(a[8], &plain), C = num(a[9], &plain), H = num(a[10], &plain), W = num(a[11], &plain), layout = name(g_layouts, a[12], &plain), K = num(a[13], &plain);
    const int dtype = name(g_dtypes, a[14], &plain);
    const float* mean_lo = ptr(a[15], &plain);
    void* ws = ptr(a[16], &plain);
    const size_t bytes = room(a[16], a[17], &plain);
    void* st = stream(a[18], &plain);
    CALL(g_backward(dy, x, mean, invstd, gamma, dx, dgamma, dbeta, N, C, H, W, layout, K, dtype, mean_lo, ws, bytes, st));
}
static PyObject* backward_relu(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    ARGS(21)
    const void *dy = ptr(a[0], &plain), *y = ptr(a[1], &plain), *x = ptr(a[2], &plain);
    const float *mean = ptr(a[3], &plain), *invstd = ptr(a[4], &plain), *gamma = ptr(a[5], &plain);
    void *dx = ptr(a[6], &plain), *dshortcut = ptr(a[7], &plain);
    float *dgamma = ptr(a[8], &plain), *dbeta = ptr(a[9], &plain);
    const int N = num(a[10], &plain), C = num(a[11], &plain), H = num(a[12], &plain), W = num(a[13], &plain), layout = name(g_layouts, a[14], &plain), K = num(a[15], &plain);
    const int dtype = name(g_dtypes, a[16], &plain);
    const float* mean_lo = ptr(a[17], &plain);
    void* ws = ptr(a[18], &plain);
    const size_t bytes = room(a[18], a[19], &plain);
    void* st = stream(a[20], &plain);
    CALL(g_backward_relu(dy, y, x, mean, invstd, gamma, dx, dshortcut, dgamma, dbeta, N, C, H, W, layout, K, dtype, mean_lo, ws, bytes, st));
}
static PyObject* frozen_forward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    ARGS(14)
    const void* x = ptr(a[0], &plain);
    const int N = num(a[1], &plain), C = num(a[2], &plain), H = num(a[3], &plain), W = num(a[4], &plain), layout = name(g_layouts, a[5], &plain), dtype = name(g_dtypes, a[6], &plain);
    const float *fixed_mean = ptr(a[7], &plain), *fixed_var = ptr(a[8], &plain), *gamma = ptr(a[9], &plain), *beta = ptr(a[10], &plain);
    const float eps = real(a[11], &plain);
    void* y = ptr(a[12], &plain);
    void* st = stream(a[13], &plain);
    CALL(g_frozen_forward(x, N, C, H, W, layout, dtype, fixed_mean, fixed_var, gamma, beta, eps, y, st));
}
static PyObject* frozen_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    ARGS(12)
    const void* dy = ptr(a[0], &plain);
    const int N = num(a[1], &plain), C = num(a[2], &plain), H = num(a[3], &plain), W = num(a[4], &plain), layout = name(g_layouts, a[5], &plain), dtype = name(g_dtypes, a[6], &plain);
    const float *fixed_var = ptr(a[7], &plain), *gamma = ptr(a[8], &plain);
    const float eps = real(a[9], &plain);
    void* dx = ptr(a[10], &plain);
    void* st = stream(a[11], &plain);
    CALL(g_frozen_backward(dy, N, C, H, W, layout, dtype, fixed_var, gamma, eps, dx, st));
}

#define LAYER_ARGS(count_)                                                                               \
    ARGS(count_)                                                                                         \
    if (!g_linear_forward) { PyErr_SetString(PyExc_RuntimeError, "bind_layers() first"); return NULL; }

static PyObject* linear_forward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    LAYER_ARGS(14)
    const void *x = ptr(a[0], &plain), *w = ptr(a[1], &plain);
    const float* bias = ptr(a[2], &plain);
    const void* residual = ptr(a[3], &plain);
    const long long M = wide(a[4], &plain);
    const int N = num(a[5], &plain), K = num(a[6], &plain), act = name(g_activations, a[7], &plain);
    void *y = ptr(a[8], &plain), *z = ptr(a[9], &plain);
    const int dtype = name(g_dtypes, a[10], &plain);
    void* ws = ptr(a[11], &plain);
    const size_t bytes = room(a[11], a[12], &plain);
    void* st = stream(a[13], &plain);
    CALL(g_linear_forward(x, w, bias, residual, M, N, K, act, y, z, dtype, ws, bytes, st));
}
static PyObject* linear_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    LAYER_ARGS(16)
    const void *dy = ptr(a[0], &plain), *x = ptr(a[1], &plain), *w = ptr(a[2], &plain), *saved = ptr(a[3], &plain);
    const long long M = wide(a[4], &plain);
    const int N = num(a[5], &plain), K = num(a[6], &plain), act = name(g_activations, a[7], &plain);
    void *dx = ptr(a[8], &plain), *dw = ptr(a[9], &plain);
    float* dbias = ptr(a[10], &plain);
    void* dresidual = ptr(a[11], &plain);
    const int dtype = name(g_dtypes, a[12], &plain);
    void* ws = ptr(a[13], &plain);
    const size_t bytes = room(a[13], a[14], &plain);
    void* st = stream(a[15], &plain);
    CALL(g_linear_backward(dy, x, w, saved, M, N, K, act, dx, dw, dbias, dresidual, dtype, ws, bytes, st));
}
static PyObject* gated_forward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    LAYER_ARGS(14)
    const void *x = ptr(a[0], &plain), *wg = ptr(a[1], &plain), *wu = ptr(a[2], &plain);
    const long long M = wide(a[3], &plain);
    const int F = num(a[4], &plain), K = num(a[5], &plain), act = name(g_activations, a[6], &plain);
    void *h = ptr(a[7], &plain), *gate = ptr(a[8], &plain), *up = ptr(a[9], &plain);
    const int dtype = name(g_dtypes, a[10], &plain);
    void* ws = ptr(a[11], &plain);
    const size_t bytes = room(a[11], a[12], &plain);
    void* st = stream(a[13], &plain);
    CALL(g_gated_forward(x, wg, wu, M, F, K, act, h, gate, up, dtype, ws, bytes, st));
}
static PyObject* gated_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    LAYER_ARGS(17)
    const void *dh = ptr(a[0], &plain), *x = ptr(a[1], &plain), *wg = ptr(a[2], &plain), *wu = ptr(a[3], &plain), *gate = ptr(a[4], &plain), *up = ptr(a[5], &plain);
    const long long M = wide(a[6], &plain);
    const int F = num(a[7], &plain), K = num(a[8], &plain), act = name(g_activations, a[9], &plain);
    void *dx = ptr(a[10], &plain), *dwg = ptr(a[11], &plain), *dwu = ptr(a[12], &plain);
    const int dtype = name(g_dtypes, a[13], &plain);
    void* ws = ptr(a[14], &plain);
    const size_t bytes = room(a[14], a[15], &plain);
    void* st = stream(a[16], &plain);
    CALL(g_gated_backward(dh, x, wg, wu, gate, up, M, F, K, act, dx, dwg, dwu, dtype, ws, bytes, st));
}
static PyObject* head_norm_forward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    LAYER_ARGS(23)
    const void* q = ptr(a[0], &plain);
    const long long ldq = wide(a[1], &plain);
    const void* k = ptr(a[2], &plain);
    const long long ldk = wide(a[3], &plain), T = wide(a[4], &plain);
    const int Hq = num(a[5], &plain), Hk = num(a[6], &plain), D = num(a[7], &plain), R = num(a[8], &plain), style = name(g_rotations, a[9], &plain);
    const int* positions = ptr(a[10], &plain);
    const float *cosines = ptr(a[11], &plain), *sines = ptr(a[12], &plain);
    const int table = num(a[13], &plain);
    const float *wq = ptr(a[14], &plain), *wk = ptr(a[15], &plain);
    const float eps = real(a[16], &plain);
    void* yq = ptr(a[17], &plain);
    const long long ldyq = wide(a[18], &plain);
    void* yk = ptr(a[19], &plain);
    const long long ldyk = wide(a[20], &plain);
    const int dtype = name(g_dtypes, a[21], &plain);
    void* st = stream(a[22], &plain);
    CALL(g_head_norm_forward(q, ldq, k, ldk, T, Hq, Hk, D, R, style, positions, cosines, sines, table, wq, wk, eps, yq, ldyq, yk, ldyk, dtype, st));
}
static PyObject* head_norm_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    LAYER_ARGS(31)
    const void* dyq = ptr(a[0], &plain);
    const long long lddyq = wide(a[1], &plain);
    const void* dyk = ptr(a[2], &plain);
    const long long lddyk = wide(a[3], &plain);
    const void* q = ptr(a[4], &plain);
    const long long ldq = wide(a[5], &plain);
    const void* k = ptr(a[6], &plain);
    const long long ldk = wide(a[7], &plain), T = wide(a[8], &plain);
    const int Hq = num(a[9], &plain), Hk = num(a[10], &plain), D = num(a[11], &plain), R = num(a[12], &plain), style = name(g_rotations, a[13], &plain);
    const int* positions = ptr(a[14], &plain);
    const float *cosines = ptr(a[15], &plain), *sines = ptr(a[16], &plain);
    const int table = num(a[17], &plain);
    const float *wq = ptr(a[18], &plain), *wk = ptr(a[19], &plain);
    const float eps = real(a[20], &plain);
    void* dq = ptr(a[21], &plain);
    const long long lddq = wide(a[22], &plain);
    void* dk = ptr(a[23], &plain);
    const long long lddk = wide(a[24], &plain);
    float *dwq = ptr(a[25], &plain), *dwk = ptr(a[26], &plain);
    const int dtype = name(g_dtypes, a[27], &plain);
    void* ws = ptr(a[28], &plain);
    const size_t bytes = room(a[28], a[29], &plain);
    void* st = stream(a[30], &plain);
    CALL(g_head_norm_backward(dyq, lddyq, dyk, lddyk, q, ldq, k, ldk, T, Hq, Hk, D, R, style, positions, cosines, sines, table, wq, wk, eps, dq, lddq, dk,
                              lddk, dwq, dwk, dtype, ws, bytes, st));
}

#define SERVING_ARGS(count_)                                                                             \
    LAYER_ARGS(count_)                                                                                   \
    if (!g_rotate_forward) { PyErr_SetString(PyExc_RuntimeError, "bind_serving() first"); return NULL; }

static PyObject* rotate(PyObject* const* a, Py_ssize_t n, rotate_fn* fn)
{
    SERVING_ARGS(19)
    const void* q = ptr(a[0], &plain);
    const long long ldq = wide(a[1], &plain);
    const void* k = ptr(a[2], &plain);
    const long long ldk = wide(a[3], &plain), T = wide(a[4], &plain);
    const int Hq = num(a[5], &plain), Hk = num(a[6], &plain), D = num(a[7], &plain), R = num(a[8], &plain), style = name(g_rotations, a[9], &plain);
    const int* positions = ptr(a[10], &plain);
    const double* freq = ptr(a[11], &plain);
    const float magnitude = real(a[12], &plain);
    void* yq = ptr(a[13], &plain);
    const long long ldyq = wide(a[14], &plain);
    void* yk = ptr(a[15], &plain);
    const long long ldyk = wide(a[16], &plain);
    const int dtype = name(g_dtypes, a[17], &plain);
    void* st = stream(a[18], &plain);
    CALL((*fn)(q, ldq, k, ldk, T, Hq, Hk, D, R, style, positions, freq, magnitude, yq, ldyq, yk, ldyk, dtype, st));
}
static PyObject* rotate_forward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    return rotate(a, n, &g_rotate_forward);
}
static PyObject* rotate_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    return rotate(a, n, &g_rotate_backward);
}
static PyObject* page_plan(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    SERVING_ARGS(20)
    const int *have = ptr(a[0], &plain), *fresh = ptr(a[1], &plain);
    const int B = num(a[2], &plain), before = num(a[3], &plain);
    const int* free_pages = ptr(a[4], &plain);
    const int free_count = num(a[5], &plain);
    const int* taken = ptr(a[6], &plain);
    int *counts = ptr(a[7], &plain), *table = ptr(a[8], &plain);
    const int max_pages = num(a[9], &plain), pages = num(a[10], &plain), page = num(a[11], &plain);
    const long long T = wide(a[12], &plain);
    int *rows = ptr(a[13], &plain), *lengths = ptr(a[14], &plain), *slots = ptr(a[15], &plain), *positions = ptr(a[16], &plain);
    void* ws = ptr(a[17], &plain);
    const size_t bytes = room(a[17], a[18], &plain);
    void* st = stream(a[19], &plain);
    CALL(g_page_plan(have, fresh, B, before, free_pages, free_count, taken, counts, table, max_pages, pages, page, T, rows, lengths, slots, positions, ws,
                     bytes, st));
}
static PyObject* page_store(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    SERVING_ARGS(14)
    const void* k = ptr(a[0], &plain);
    const long long ldk = wide(a[1], &plain);
    const void* v = ptr(a[2], &plain);
    const long long ldv = wide(a[3], &plain), T = wide(a[4], &plain);
    const int Hk = num(a[5], &plain), D = num(a[6], &plain);
    const int* slots = ptr(a[7], &plain);
    void *k_pages = ptr(a[8], &plain), *v_pages = ptr(a[9], &plain);
    const int pages = num(a[10], &plain), page = num(a[11], &plain), dtype = name(g_dtypes, a[12], &plain);
    void* st = stream(a[13], &plain);
    CALL(g_page_store(k, ldk, v, ldv, T, Hk, D, slots, k_pages, v_pages, pages, page, dtype, st));
}
static PyObject* prefix_attention(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    SERVING_ARGS(25)
    const void* q = ptr(a[0], &plain);
    const long long ldq = wide(a[1], &plain), T = wide(a[2], &plain);
    const int B = num(a[3], &plain);
    const int *rows = ptr(a[4], &plain), *lengths = ptr(a[5], &plain);
    const int Hq = num(a[6], &plain), Hk = num(a[7], &plain), D = num(a[8], &plain);
    const float scale = real(a[9], &plain);
    const void *k_pages = ptr(a[10], &plain), *v_pages = ptr(a[11], &plain);
    const int pages = num(a[12], &plain), page = num(a[13], &plain);
    const int* prefix_table = ptr(a[14], &plain);
    const int prefix = num(a[15], &plain);
    const int* table = ptr(a[16], &plain);
    const int max_pages = num(a[17], &plain);
    void* out = ptr(a[18], &plain);
    const long long ldo = wide(a[19], &plain);
    float* lse = ptr(a[20], &plain);
    const int dtype = name(g_dtypes, a[21], &plain);
    void* ws = ptr(a[22], &plain);
    const size_t bytes = room(a[22], a[23], &plain);
    void* st = stream(a[24], &plain);
    CALL(g_prefix_attention(q, ldq, T, B, rows, lengths, Hq, Hk, D, scale, k_pages, v_pages, pages, page, prefix_table, prefix, table, max_pages, out, ldo,
                            lse, dtype, ws, bytes, st));
}

/* bind_serving(addresses of the five functions), after bind_layers() */
static PyObject* bind_serving(PyObject* self, PyObject* args)
{
    unsigned long long f[5];
    (void)self;
    if (!PyArg_ParseTuple(args, "(KKKKK)", &f[0], &f[1], &f[2], &f[3], &f[4])) return NULL;
    g_rotate_forward = (rotate_fn)(uintptr_t)f[0];
    g_rotate_backward = (rotate_fn)(uintptr_t)f[1];
    g_page_plan = (page_plan_fn)(uintptr_t)f[2];
    g_page_store = (page_store_fn)(uintptr_t)f[3];
    g_prefix_attention = (prefix_attention_fn)(uintptr_t)f[4];
    Py_RETURN_NONE;
}

/* bind_layers(addresses of the six functions of the layers, activations, rotations), after bind() */
static PyObject* bind_layers(PyObject* self, PyObject* args)
{
    unsigned long long f[6];
    PyObject *activations, *rotations;
    (void)self;
    if (!PyArg_ParseTuple(args, "(KKKKKK)OO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &activations, &rotations)) return NULL;
    Py_INCREF(activations);
    Py_INCREF(rotations);
    Py_XSETREF(g_activations, activations);
    Py_XSETREF(g_rotations, rotations);
    g_linear_forward = (linear_forward_fn)(uintptr_t)f[0];
    g_linear_backward = (linear_backward_fn)(uintptr_t)f[1];
    g_gated_forward = (gated_forward_fn)(uintptr_t)f[2];
    g_gated_backward = (gated_backward_fn)(uintptr_t)f[3];
    g_head_norm_forward = (head_norm_forward_fn)(uintptr_t)f[4];
    g_head_norm_backward = (head_norm_backward_fn)(uintptr_t)f[5];
    Py_RETURN_NONE;
}

/* bind(addresses of the six functions, layouts, dtypes, stream) */
static PyObject* bind(PyObject* self, PyObject* args)
{
    unsigned long long f[6];
    PyObject *layouts, *dtypes, *st;
    (void)self;
    if (!PyArg_ParseTuple(args, "(KKKKKK)OOO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &layouts, &dtypes, &st)) return NULL;
    Py_INCREF(layouts);
    Py_INCREF(dtypes);
    Py_INCREF(st);
    Py_XSETREF(g_layouts, layouts);
    Py_XSETREF(g_dtypes, dtypes);
    Py_XSETREF(g_stream, st);
    g_forward = (forward_fn)(uintptr_t)f[0];
    g_forward_relu = (forward_relu_fn)(uintptr_t)f[1];
    g_backward = (backward_fn)(uintptr_t)f[2];
    g_backward_relu = (backward_relu_fn)(uintptr_t)f[3];
    g_frozen_forward = (frozen_forward_fn)(uintptr_t)f[4];
    g_frozen_backward = (frozen_backward_fn)(uintptr_t)f[5];
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, NULL},
    {"forward", (PyCFunction)(void (*)(void))forward, METH_FASTCALL, NULL},
    {"forward_relu", (PyCFunction)(void (*)(void))forward_relu, METH_FASTCALL, NULL},
    {"backward", (PyCFunction)(void (*)(void))backward, METH_FASTCALL, NULL},
    {"backward_relu", (PyCFunction)(void (*)(void))backward_relu, METH_FASTCALL, NULL},
    {"frozen_forward", (PyCFunction)(void (*)(void))frozen_forward, METH_FASTCALL, NULL},
    {"frozen_backward", (PyCFunction)(void (*)(void))frozen_backward, METH_FASTCALL, NULL},
    {"bind_layers", bind_layers, METH_VARARGS, NULL},
    {"linear_forward", (PyCFunction)(void (*)(void))linear_forward, METH_FASTCALL, NULL},
    {"linear_backward", (PyCFunction)(void (*)(void))linear_backward, METH_FASTCALL, NULL},
    {"gated_forward", (PyCFunction)(void (*)(void))gated_forward, METH_FASTCALL, NULL},
    {"gated_backward", (PyCFunction)(void (*)(void))gated_backward, METH_FASTCALL, NULL},
    {"head_norm_forward", (PyCFunction)(void (*)(void))head_norm_forward, METH_FASTCALL, NULL},
    {"head_norm_backward", (PyCFunction)(void (*)(void))head_norm_backward, METH_FASTCALL, NULL},
    {"bind_serving", bind_serving, METH_VARARGS, NULL},
    {"rotate_forward", (PyCFunction)(void (*)(void))rotate_forward, METH_FASTCALL, NULL},
    {"rotate_backward", (PyCFunction)(void (*)(void))rotate_backward, METH_FASTCALL, NULL},
    {"page_plan", (PyCFunction)(void (*)(void))page_plan, METH_FASTCALL, NULL},
    {"page_store", (PyCFunction)(void (*)(void))page_store, METH_FASTCALL, NULL},
    {"prefix_attention", (PyCFunction)(void (*)(void))prefix_attention, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cgbn_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__cgbn_call(void)
{
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_numel = PyUnicode_InternFromString("numel");
    g_element_size = PyUnicode_InternFromString("element_size");
    if (!g_data_ptr || !g_numel || !g_element_size) return NULL;
    return PyModule_Create(&module);
}
