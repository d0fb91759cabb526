// The calls on rows from Python, in C++: arguments of torch tensors straight into the C interface's structures.  A small call's time
// is that of the host: through the ctypes binding 3.6 us of a product's 6.4 went into asking tensors for their shape and address.
//
// Each function returns the call's status, or -1 where an argument is anything but an ordinary tensor that the call takes as it is;
// gdws.py then goes through the same checks one by one and says what is wrong, or takes the call itself.  So it does where torch
// throws: the tensors of a functional transform (vmap, grad) have the ordinary type but no memory of their own.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include "gdws.h"

namespace {

decltype(&gdws_quantize_rows) g_quantize;
decltype(&gdws_norm_quantize_rows) g_norm;
decltype(&gdws_dequantize_rows) g_values;
decltype(&gdws_pointwise8) g_product;
PyObject *g_device, *g_stream;       // torch's current device; its current stream of a device, as an integer

const at::Tensor *tensor(PyObject *o, long device)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.has_storage() && t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided && !t.is_conj() && !t.is_neg() ? &t : nullptr;
}

bool geometry(const at::Tensor &t, int64_t *rows, int64_t *ld, int *cols)
{
    if (t.dim() != 2 || t.size(1) > 0x7fffffff || (t.stride(1) != 1 && t.size(1) > 1)) return false;
    *rows = t.size(0); *ld = t.stride(0); *cols = (int)t.size(1);
    return true;
}

bool type_of(const at::Tensor &t, gdws_dtype_t *type)
{
    const auto s = t.scalar_type();
    *type = s == at::kFloat ? GDWS_F32 : GDWS_BF16;
    return s == at::kFloat || s == at::kBFloat16;
}

bool values(PyObject *o, long device, gdws_rows_t *m)
{
    const at::Tensor *t = tensor(o, device);
    if (!t || !type_of(*t, &m->dtype) || !geometry(*t, &m->rows, &m->ld, &m->cols)) return false;
    m->ptr = t->data_ptr();
    return true;
}

const at::Tensor *vector(PyObject *o, long device, int64_t n)
{
    const at::Tensor *t = tensor(o, device);
    return t && t->numel() == n && t->is_contiguous() ? t : nullptr;
}

bool steps(PyObject *q, PyObject *scale, long device, gdws_rows8_t *m)
{
    const at::Tensor *t = tensor(q, device);
    if (!t || t->scalar_type() != at::kChar || !geometry(*t, &m->rows, &m->ld, &m->cols)) return false;
    const at::Tensor *s = vector(scale, device, m->rows);
    if (!s || s->scalar_type() != at::kFloat) return false;
    m->q = (int8_t *)t->data_ptr();
    m->scale = (float *)s->data_ptr();
    return true;
}

// The current device and its stream; false: a Python error is set.
bool place(long *device, void **stream)
{
    PyObject *d = PyObject_CallNoArgs(g_device);
    if (!d) return false;
    *device = PyLong_AsLong(d);
    PyObject *s = *device < 0 && PyErr_Occurred() ? nullptr : PyObject_CallOneArg(g_stream, d);
    Py_DECREF(d);
    if (!s) return false;
    *stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    return !PyErr_Occurred();
}

struct WithoutGil {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};
template <class Call>
PyObject *status_of(Call call)
{
    gdws_status_t st;
    {
        WithoutGil released;
        st = call();
    }
    return PyLong_FromLong((long)st);
}
PyObject *other() { return PyLong_FromLong(-1); }

PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 6) return PyErr_Format(PyExc_TypeError, "bind takes four addresses and two functions");
    g_quantize = (decltype(g_quantize))PyLong_AsVoidPtr(a[0]);
    g_norm = (decltype(g_norm))PyLong_AsVoidPtr(a[1]);
    g_values = (decltype(g_values))PyLong_AsVoidPtr(a[2]);
    g_product = (decltype(g_product))PyLong_AsVoidPtr(a[3]);
    if (PyErr_Occurred()) return nullptr;
    Py_INCREF(a[4]); Py_INCREF(a[5]);
    Py_XDECREF(g_device); Py_XDECREF(g_stream);
    g_device = a[4]; g_stream = a[5];
    Py_RETURN_NONE;
}

bool ready(Py_ssize_t n, Py_ssize_t want) { return n == want && g_device; }

PyObject *quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n)              // x, q, scale
{
    long device;
    void *stream;
    gdws_rows_t x;
    gdws_rows8_t q;
    if (!ready(n, 3)) return other();
    if (!place(&device, &stream)) return nullptr;
    if (!values(a[0], device, &x) || !steps(a[1], a[2], device, &q)) return other();
    return status_of([&] { return g_quantize(&x, &q, stream); });
}

PyObject *dequantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n)            // q, scale, y
{
    long device;
    void *stream;
    gdws_rows_t y;
    gdws_rows8_t q;
    if (!ready(n, 3)) return other();
    if (!place(&device, &stream)) return nullptr;
    if (!values(a[2], device, &y) || !steps(a[0], a[1], device, &q)) return other();
    return status_of([&] { return g_values(&q, &y, stream); });
}

PyObject *norm_quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n)         // x, q, scale, weight, eps, residual, total
{
    long device;
    void *stream;
    gdws_rows_t x, residual, total;
    gdws_rows8_t q;
    gdws_dtype_t wtype = GDWS_F32;
    const void *weight = nullptr;
    if (!ready(n, 7) || !PyFloat_CheckExact(a[4])) return other();
    if (!place(&device, &stream)) return nullptr;
    const bool has_residual = a[5] != Py_None, has_total = a[6] != Py_None;
    if (!values(a[0], device, &x) || !steps(a[1], a[2], device, &q) || (has_residual && !values(a[5], device, &residual)) || (has_total && !values(a[6], device, &total))) return other();
    if (a[3] != Py_None) {
        const at::Tensor *w = vector(a[3], device, x.cols);
        if (!w || !type_of(*w, &wtype)) return other();
        weight = w->data_ptr();
    }
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    return status_of([&] { return g_norm(&x, has_residual ? &residual : nullptr, has_total ? &total : nullptr, weight, wtype, eps, &q, stream); });
}

PyObject *pointwise8(PyObject *, PyObject *const *a, Py_ssize_t n)                 // q, scale, w, w_scale, y, bias, relu
{
    long device;
    void *stream;
    gdws_rows_t y;
    gdws_rows8_t x, w;
    const float *bias = nullptr;
    if (!ready(n, 7)) return other();
    if (!place(&device, &stream)) return nullptr;
    if (!steps(a[0], a[1], device, &x) || !steps(a[2], a[3], device, &w) || !values(a[4], device, &y)) return other();
    if (a[5] != Py_None) {
        const at::Tensor *b = vector(a[5], device, y.cols);
        if (!b || b->scalar_type() != at::kFloat) return other();
        bias = (const float *)b->data_ptr();
    }
    const int relu = PyObject_IsTrue(a[6]);
    if (relu < 0) return nullptr;
    return status_of([&] { return g_product(&x, &w, bias, relu, &y, stream); });
}

// Nothing is thrown into the interpreter, which is C.
template <PyObject *(*function)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    try {
        return function(self, a, n);
    } catch (...) {
        PyErr_Clear();
        return other();
    }
}
template <PyObject *(*function)(PyObject *, PyObject *const *, Py_ssize_t)>
PyCFunction method() { return (PyCFunction)(void (*)(void))guarded<function>; }

PyMethodDef g_methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"quantize_rows", method<quantize_rows>(), METH_FASTCALL, nullptr},
    {"dequantize_rows", method<dequantize_rows>(), METH_FASTCALL, nullptr},
    {"norm_quantize_rows", method<norm_quantize_rows>(), METH_FASTCALL, nullptr},
    {"pointwise8", method<pointwise8>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows(void)
{
    PyObject *m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}
