// What the binding asks of tensors, as an extension module: checks, addresses and strides.  A call of the reading step takes up
// to a dozen tensors and some microseconds; asked from Python, each tensor costs a third of a microsecond, here a tenth of
// that.  Errors are raised here; no tensor is kept.
#define PY_SSIZE_T_CLEAN   // (before any header of Python)
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include "pq_read.h"

namespace {

const char *dtype_name(at::ScalarType t) { return c10::toString(t); }

// The tensor behind an object, or null with an error set.
const at::Tensor *tensor_of(PyObject *o, const char *name) {
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%s must be a GPU tensor", name);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

bool has_dtype(const at::Tensor &t, PyObject *dtype, const char *name) {
    if (!THPDtype_Check(dtype)) {
        PyErr_SetString(PyExc_TypeError, "not a dtype");
        return false;
    }
    const at::ScalarType want = ((THPDtype *)dtype)->scalar_type;
    if (t.scalar_type() == want) return true;
    PyErr_Format(PyExc_TypeError, "%s must have dtype %s, got %s", name, dtype_name(want), dtype_name(t.scalar_type()));
    return false;
}

bool has_shape(const at::Tensor &t, PyObject *shape, const char *name) {
    if (PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == t.dim()) {
        bool same = true;
        for (int64_t i = 0; i < t.dim() && same; ++i) same = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)) == t.size(i);
        if (same) return true;
        if (PyErr_Occurred()) return false;
    }
    PyErr_Format(PyExc_ValueError, "%s does not have shape %R", name, shape);
    return false;
}

bool rows_contiguous(const at::Tensor &t, const char *name) {
    const int64_t last = t.dim() - 1;
    if (t.stride(last) == 1 || t.size(last) <= 1 || t.numel() == 0) return true;
    PyErr_Format(PyExc_ValueError, "the elements of a row of %s must be contiguous", name);
    return false;
}

int elem_of(const at::Tensor &t, const char *name) {
    switch (t.scalar_type()) {
    case at::kFloat: return PQ_ELEM_F32;
    case at::kHalf: return PQ_ELEM_F16;
    case at::kBFloat16: return PQ_ELEM_BF16;
    default: PyErr_Format(PyExc_TypeError, "%s has dtype %s: float32, float16 or bfloat16", name, dtype_name(t.scalar_type())); return -1;
    }
}

// address(tensor, dtype, name, shape): of a contiguous tensor that the library reads and writes where it lies; None of None
PyObject *address(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "address takes a tensor, a dtype, a name and a shape");
    if (args[0] == Py_None) Py_RETURN_NONE;
    const char *name = PyUnicode_AsUTF8(args[2]);
    const at::Tensor *t = name ? tensor_of(args[0], name) : nullptr;
    if (!t || !has_dtype(*t, args[1], name)) return nullptr;
    if (!t->is_contiguous()) return PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
    if (!has_shape(*t, args[3], name)) return nullptr;
    return PyLong_FromVoidPtr(t->data_ptr());
}

// heads(tensor, dtype, name, shape): rows [tokens][heads][dim] of any strides but the last, as the bytes of a pq_heads
PyObject *heads(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "heads takes a tensor, a dtype, a name and a shape");
    const char *name = PyUnicode_AsUTF8(args[2]);
    const at::Tensor *t = name ? tensor_of(args[0], name) : nullptr;
    if (!t || !has_dtype(*t, args[1], name) || !has_shape(*t, args[3], name) || !rows_contiguous(*t, name)) return nullptr;
    const pq_heads h = {t->data_ptr(), t->stride(0), t->stride(1)};
    return PyBytes_FromStringAndSize((const char *)&h, sizeof(h));
}

// rows(tensor, name): a matrix of any strides but the last -> (address, pq_elem, row stride, rows, columns)
PyObject *rows(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 2) return PyErr_Format(PyExc_TypeError, "rows takes a tensor and a name");
    const char *name = PyUnicode_AsUTF8(args[1]);
    const at::Tensor *t = name ? tensor_of(args[0], name) : nullptr;
    if (!t) return nullptr;
    const int elem = elem_of(*t, name);
    if (elem < 0) return nullptr;
    if (t->dim() != 2) return PyErr_Format(PyExc_ValueError, "%s must be a matrix", name);
    if (!rows_contiguous(*t, name)) return nullptr;
    return Py_BuildValue("KiLLL", (unsigned long long)(uintptr_t)t->data_ptr(), elem, (long long)t->stride(0), (long long)t->size(0), (long long)t->size(1));
}

// cache(keys, values): paged [blocks][block size][heads][dim] of any strides but the last -> (bytes of a pq_kv_cache, heads, dim)
PyObject *cache(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 2) return PyErr_Format(PyExc_TypeError, "cache takes keys and values");
    const at::Tensor *k = tensor_of(args[0], "key_cache"), *v = k ? tensor_of(args[1], "value_cache") : nullptr;
    if (!v) return nullptr;
    const int elem = elem_of(*k, "key_cache");
    if (elem < 0) return nullptr;
    if (v->scalar_type() != k->scalar_type())
        return PyErr_Format(PyExc_TypeError, "value_cache has dtype %s, key_cache %s", dtype_name(v->scalar_type()), dtype_name(k->scalar_type()));
    if (k->dim() != 4 || !v->sizes().equals(k->sizes()))
        return PyErr_Format(PyExc_ValueError, "keys and values must have one shape [blocks][block size][heads][dim]");
    if (!rows_contiguous(*k, "key_cache") || !rows_contiguous(*v, "value_cache")) return nullptr;
    if (k->size(1) > INT32_MAX || k->size(2) > INT32_MAX || k->size(3) > INT32_MAX) return PyErr_Format(PyExc_ValueError, "the cache is too large");
    pq_kv_cache c = {k->data_ptr(), v->data_ptr(), {k->stride(0), k->stride(1), k->stride(2)}, {v->stride(0), v->stride(1), v->stride(2)},
                     k->size(0), (int)k->size(1), (int)k->size(2), (int)k->size(3), (pq_elem)elem};
    return Py_BuildValue("y#ii", (const char *)&c, (Py_ssize_t)sizeof(c), c.heads, c.dim);
}

typedef PyObject *(*fast_function)(PyObject *, PyObject *const *, Py_ssize_t);
template <fast_function F> PyObject *guarded(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    try {
        return F(self, args, n);
    } catch (const std::exception &e) {   // (tensors without storage and the like)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {{"address", (PyCFunction)(void (*)())(fast_function)guarded<address>, METH_FASTCALL, nullptr},
                         {"heads", (PyCFunction)(void (*)())(fast_function)guarded<heads>, METH_FASTCALL, nullptr},
                         {"rows", (PyCFunction)(void (*)())(fast_function)guarded<rows>, METH_FASTCALL, nullptr},
                         {"cache", (PyCFunction)(void (*)())(fast_function)guarded<cache>, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tensor_views", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_tensor_views(void) { return PyModule_Create(&module); }
