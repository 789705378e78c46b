// The calls of the reading step from Python, as an extension module: checks of the tensors, their addresses and strides, and the
// library's function.  A call takes up to a dozen tensors, and where tokens are few its kernel takes less than these do if they are
// asked from Python: the plan of 64 requests 5.0 us a call by way of Python's foreign functions, 3.5 us from here; the append of
// 64 tokens 5.9 and 3.8 us.  Errors are raised here; no tensor is kept.
#define PY_SSIZE_T_CLEAN   // (before any header of Python)
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <string>

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

// Paged [blocks][block size][heads][dim] of any strides but the last.
bool read_cache(PyObject *keys, PyObject *values, pq_kv_cache *c) {
    const at::Tensor *k = tensor_of(keys, "key_cache"), *v = k ? tensor_of(values, "value_cache") : nullptr;
    if (!v) return false;
    const int elem = elem_of(*k, "key_cache");
    if (elem < 0) return false;
    if (v->scalar_type() != k->scalar_type()) {
        PyErr_Format(PyExc_TypeError, "value_cache has dtype %s, key_cache %s", dtype_name(v->scalar_type()), dtype_name(k->scalar_type()));
        return false;
    }
    if (k->dim() != 4 || !v->sizes().equals(k->sizes())) {
        PyErr_Format(PyExc_ValueError, "keys and values must have one shape [blocks][block size][heads][dim]");
        return false;
    }
    if (!rows_contiguous(*k, "key_cache") || !rows_contiguous(*v, "value_cache")) return false;
    if (k->size(1) > INT32_MAX || k->size(2) > INT32_MAX || k->size(3) > INT32_MAX) {
        PyErr_Format(PyExc_ValueError, "the cache is too large");
        return false;
    }
    *c = {k->data_ptr(), v->data_ptr(), {k->stride(0), k->stride(1), k->stride(2)}, {v->stride(0), v->stride(1), v->stride(2)},
          k->size(0), (int)k->size(1), (int)k->size(2), (int)k->size(3), (pq_elem)elem};
    return true;
}

bool has_type(const at::Tensor &t, at::ScalarType want, const char *name) {
    if (t.scalar_type() == want) return true;
    PyErr_Format(PyExc_TypeError, "%s must have dtype %s, got %s", name, dtype_name(want), dtype_name(t.scalar_type()));
    return false;
}
bool has_sizes(const at::Tensor &t, at::IntArrayRef want, const char *name) {
    if (t.sizes().equals(want)) return true;
    std::string text;
    for (const int64_t n : want) text += (text.empty() ? "" : ", ") + std::to_string(n);
    PyErr_Format(PyExc_ValueError, "%s does not have shape (%s)", name, text.c_str());
    return false;
}
// The address of a contiguous tensor of that type and shape (null of None, where that may be).
template <class P> bool in_place(PyObject *o, at::ScalarType type, at::IntArrayRef sizes, const char *name, P **p, bool may_be_none = false) {
    *p = nullptr;
    if (may_be_none && o == Py_None) return true;
    const at::Tensor *t = tensor_of(o, name);
    if (!t || !has_type(*t, type, name)) return false;
    if (!t->is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
        return false;
    }
    if (!has_sizes(*t, sizes, name)) return false;
    *p = (P *)t->data_ptr();
    return true;
}
// Rows [tokens][heads][dim] of any strides but the last.
bool in_rows(PyObject *o, at::ScalarType type, at::IntArrayRef sizes, const char *name, pq_heads *h) {
    const at::Tensor *t = tensor_of(o, name);
    if (!t || !has_type(*t, type, name) || !has_sizes(*t, sizes, name) || !rows_contiguous(*t, name)) return false;
    *h = {t->data_ptr(), t->stride(0), t->stride(1)};
    return true;
}
bool whole(PyObject *o, int64_t *x) {
    *x = PyLong_AsLongLong(o);
    return *x != -1 || !PyErr_Occurred();
}
// The library's function and context, as the binding has them: addresses (a closed context's is None: the library refuses it).
template <class F> bool entry(PyObject *const *args, F **f, pq_ctx **ctx) {
    *f = (F *)PyLong_AsVoidPtr(args[0]);
    *ctx = !*f || args[1] == Py_None ? nullptr : (pq_ctx *)PyLong_AsVoidPtr(args[1]);
    if (*f && (*ctx || !PyErr_Occurred())) return true;
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no function");
    return false;
}
template <class F> PyObject *without_gil(F f) {
    PyThreadState *const state = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(state);
    return PyLong_FromLong(rc);
}

// plan(function, context, new_lens, cached_lens, block_tables, free_blocks, block_size, ntokens, cu_new, kv_lens, positions, slots, taken)
PyObject *plan(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 13) return PyErr_Format(PyExc_TypeError, "plan takes 13 arguments");
    decltype(pq_kv_plan) *f;
    pq_ctx *ctx;
    int64_t block_size, ntokens;
    if (!entry(args, &f, &ctx) || !whole(args[6], &block_size) || !whole(args[7], &ntokens)) return nullptr;
    const at::Tensor *tables = tensor_of(args[4], "block_tables"), *free_blocks = tables ? tensor_of(args[5], "free_blocks") : nullptr;
    if (!free_blocks) return nullptr;
    if (tables->dim() != 2) return PyErr_Format(PyExc_ValueError, "block_tables must be [requests][width]");
    const int64_t nreq = tables->size(0), width = tables->size(1), nfree = free_blocks->numel();
    for (const int64_t x : {nreq, width, nfree, block_size})
        if (x > INT32_MAX || x < INT32_MIN) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
    const int32_t *new_lens, *cached_lens, *free_p;
    int32_t *tables_p, *cu, *kv, *positions, *taken;
    int64_t *slots;
    // (a negative ntokens is the library's to refuse)
    const int64_t rows = std::max<int64_t>(ntokens, 0);
    if (!in_place(args[2], at::kInt, {nreq}, "new_lens", &new_lens) || !in_place(args[3], at::kInt, {nreq}, "cached_lens", &cached_lens) ||
        !in_place(args[4], at::kInt, {nreq, width}, "block_tables", &tables_p) || !in_place(args[5], at::kInt, {nfree}, "free_blocks", &free_p) ||
        !in_place(args[8], at::kInt, {nreq + 1}, "cu_new", &cu) || !in_place(args[9], at::kInt, {nreq}, "kv_lens", &kv) ||
        !in_place(args[10], at::kInt, {rows}, "positions", &positions) || !in_place(args[11], at::kLong, {rows}, "slots", &slots) ||
        !in_place(args[12], at::kInt, {1}, "taken", &taken))
        return nullptr;
    return without_gil([&] {
        return f(ctx, new_lens, cached_lens, (int)nreq, tables_p, (int)width, free_p, (int)nfree, (int)block_size, ntokens, cu, kv, positions, slots, taken);
    });
}

// append(function, context, q, k, v, positions, slots, key_cache, value_cache, cos, sin, q_weight, k_weight, eps, norm, pairs, out)
PyObject *append(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 17) return PyErr_Format(PyExc_TypeError, "append takes 17 arguments");
    decltype(pq_kv_append) *f;
    pq_ctx *ctx;
    pq_kv_cache cache;
    if (!entry(args, &f, &ctx) || !read_cache(args[7], args[8], &cache)) return nullptr;
    const at::ScalarType type = THPVariable_Unpack(args[7]).scalar_type();
    const at::Tensor *k = tensor_of(args[3], "k");
    if (!k) return nullptr;
    const int64_t t = k->dim() > 0 ? k->size(0) : 0;
    int64_t q_heads = 0, max_positions = 0, half = 0;
    pq_heads q_rows = {}, k_rows, v_rows;
    void *out = nullptr;
    if (args[2] != Py_None) {
        const at::Tensor *q = tensor_of(args[2], "q");
        if (!q) return nullptr;
        q_heads = q->dim() == 3 ? q->size(1) : 0;
        if (q_heads > INT32_MAX) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
        if (!in_rows(args[2], type, {t, q_heads, cache.dim}, "q", &q_rows) || !in_place(args[16], type, {t, q_heads, cache.dim}, "out", &out)) return nullptr;
    }
    if ((args[9] == Py_None) != (args[10] == Py_None)) return PyErr_Format(PyExc_ValueError, "cos and sin go together");
    if (args[9] != Py_None) {
        const at::Tensor *cos = tensor_of(args[9], "cos");
        if (!cos) return nullptr;
        if (cos->dim() != 2 || cos->size(1) > INT32_MAX / 2) return PyErr_Format(PyExc_ValueError, "cos and sin must be [positions][rot/2]");
        max_positions = cos->size(0);
        half = cos->size(1);
    }
    const int32_t *positions;
    const int64_t *slots;
    const float *cos_p, *sin_p, *q_weight, *k_weight;
    if (!in_rows(args[3], type, {t, cache.heads, cache.dim}, "k", &k_rows) || !in_rows(args[4], type, {t, cache.heads, cache.dim}, "v", &v_rows) ||
        !in_place(args[5], at::kInt, {t}, "positions", &positions) || !in_place(args[6], at::kLong, {t}, "slots", &slots) ||
        !in_place(args[9], at::kFloat, {max_positions, half}, "cos", &cos_p, true) || !in_place(args[10], at::kFloat, {max_positions, half}, "sin", &sin_p, true) ||
        !in_place(args[11], at::kFloat, {cache.dim}, "q_weight", &q_weight, true) || !in_place(args[12], at::kFloat, {cache.dim}, "k_weight", &k_weight, true))
        return nullptr;
    const double eps = PyFloat_AsDouble(args[13]);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    const int norm = PyObject_IsTrue(args[14]), pairs = PyObject_IsTrue(args[15]);
    if (norm < 0 || pairs < 0) return nullptr;
    return without_gil([&] {
        return f(ctx, &cache, q_heads > 0 ? &q_rows : nullptr, (int)q_heads, &k_rows, &v_rows, t, positions, slots, cos_p, sin_p, max_positions, (int)(2 * half), pairs,
                 norm, q_weight, k_weight, (float)eps, out);
    });
}

// attention(function, context, q, key_cache, value_cache, block_tables, cu_new, kv_lens, max_new, scale, window, out, lse)
PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 13) return PyErr_Format(PyExc_TypeError, "attention takes 13 arguments");
    decltype(pq_kv_attention) *f;
    pq_ctx *ctx;
    pq_kv_cache cache;
    int64_t max_new, window;
    if (!entry(args, &f, &ctx) || !read_cache(args[3], args[4], &cache) || !whole(args[8], &max_new) || !whole(args[10], &window)) return nullptr;
    const at::ScalarType type = THPVariable_Unpack(args[3]).scalar_type();
    const at::Tensor *q = tensor_of(args[2], "q"), *tables = q ? tensor_of(args[5], "block_tables") : nullptr;
    if (!tables) return nullptr;
    if (tables->dim() != 2) return PyErr_Format(PyExc_ValueError, "block_tables must be [requests][width]");
    const int64_t t = q->dim() == 3 ? q->size(0) : 0, q_heads = q->dim() == 3 ? q->size(1) : 0, nreq = tables->size(0), width = tables->size(1);
    for (const int64_t x : {q_heads, nreq, width, max_new, window})
        if (x > INT32_MAX || x < INT32_MIN) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
    const double scale = args[9] == Py_None ? 1.0 / std::sqrt((double)cache.dim) : PyFloat_AsDouble(args[9]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    pq_heads q_rows;
    const int32_t *tables_p, *cu, *kv;
    void *out;
    float *lse;
    if (!in_rows(args[2], type, {t, q_heads, cache.dim}, "q", &q_rows) || !in_place(args[5], at::kInt, {nreq, width}, "block_tables", &tables_p) ||
        !in_place(args[6], at::kInt, {nreq + 1}, "cu_new", &cu) || !in_place(args[7], at::kInt, {nreq}, "kv_lens", &kv) ||
        !in_place(args[11], type, {t, q_heads, cache.dim}, "out", &out) || !in_place(args[12], at::kFloat, {t, q_heads}, "lse", &lse))
        return nullptr;
    return without_gil([&] {
        return f(ctx, &cache, &q_rows, (int)q_heads, t, cu, kv, (int)nreq, tables_p, (int)width, (int)max_new, (float)scale, (int)window, out, lse);
    });
}

// sample(function, context, logits, noise, temperature, top_k, top_p, min_p, tokens, logprobs)
PyObject *sample(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 10) return PyErr_Format(PyExc_TypeError, "sample takes 10 arguments");
    decltype(pq_sample_tokens) *f;
    pq_ctx *ctx;
    if (!entry(args, &f, &ctx)) return nullptr;
    const at::Tensor *logits = tensor_of(args[2], "logits");
    if (!logits) return nullptr;
    const int elem = elem_of(*logits, "logits");
    if (elem < 0) return nullptr;
    if (logits->dim() != 2) return PyErr_Format(PyExc_ValueError, "logits must be [rows][vocab]");
    if (!rows_contiguous(*logits, "logits")) return nullptr;
    const int64_t rows = logits->size(0), vocab = logits->size(1);
    if (rows > INT32_MAX || vocab > INT32_MAX) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
    const float *noise = nullptr;
    int64_t noise_stride = 0;
    if (args[3] != Py_None) {
        const at::Tensor *u = tensor_of(args[3], "noise");
        if (!u || !has_type(*u, at::kFloat, "noise") || !has_sizes(*u, {rows, vocab}, "noise") || !rows_contiguous(*u, "noise")) return nullptr;
        noise = (const float *)u->data_ptr();
        noise_stride = u->stride(0);
    }
    const float *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int64_t *tokens;
    float *logprobs;
    if (!in_place(args[4], at::kFloat, {rows}, "temperature", &temperature, true) || !in_place(args[5], at::kInt, {rows}, "top_k", &top_k, true) ||
        !in_place(args[6], at::kFloat, {rows}, "top_p", &top_p, true) || !in_place(args[7], at::kFloat, {rows}, "min_p", &min_p, true) ||
        !in_place(args[8], at::kLong, {rows}, "tokens", &tokens) || !in_place(args[9], at::kFloat, {rows}, "logprobs", &logprobs, true))
        return nullptr;
    const void *const p = logits->data_ptr();
    const int64_t row_stride = logits->stride(0);
    return without_gil([&] {
        return f(ctx, p, (pq_elem)elem, row_stride, (int)rows, (int)vocab, noise, noise_stride, temperature, top_k, top_p, min_p, tokens, logprobs);
    });
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

#define METHOD(f) {#f, (PyCFunction)(void (*)())(fast_function)guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(plan), METHOD(append), METHOD(attention), METHOD(sample), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tensor_views", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_tensor_views(void) { return PyModule_Create(&module); }
