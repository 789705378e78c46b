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
template <class C> bool read_layout(PyObject *keys, PyObject *values, C *c) {
    const at::Tensor *k = tensor_of(keys, "key_cache"), *v = k ? tensor_of(values, "value_cache") : nullptr;
    if (!v) return false;
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
    c->keys = k->data_ptr();
    c->values = v->data_ptr();
    for (int i = 0; i < 3; ++i) {
        c->key_strides[i] = k->stride(i);
        c->value_strides[i] = v->stride(i);
    }
    c->nblocks = k->size(0);
    c->block_size = (int)k->size(1);
    c->heads = (int)k->size(2);
    c->dim = (int)k->size(3);
    return true;
}
bool read_cache(PyObject *keys, PyObject *values, pq_kv_cache *c) {
    const at::Tensor *k = tensor_of(keys, "key_cache"), *v = k ? tensor_of(values, "value_cache") : nullptr;
    if (!v) return false;
    const int elem = elem_of(*k, "key_cache");
    if (elem < 0 || !read_layout(keys, values, c)) return false;
    c->elem = (pq_elem)elem;
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
// The same with a scale for each block and head.
bool read_cache8(PyObject *keys, PyObject *values, PyObject *key_scales, PyObject *value_scales, pq_kv_cache8 *c) {
    const at::Tensor *k = tensor_of(keys, "key_cache");
    return k && has_type(*k, at::kFloat8_e4m3fn, "key_cache") && read_layout(keys, values, c) &&
           in_place(key_scales, at::kFloat, {c->nblocks, c->heads}, "key_scales", &c->key_scales) &&
           in_place(value_scales, at::kFloat, {c->nblocks, c->heads}, "value_scales", &c->value_scales);
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

// What append and append8 take alike, in the order of append8's arguments; f: the library's function from the queries on.
struct append_objects {
    PyObject *q, *k, *v, *positions, *slots, *cos, *sin, *q_weight, *k_weight, *eps, *norm, *pairs, *out;
};
template <class F> PyObject *append_rows(const append_objects &o, const at::Tensor &k, at::ScalarType type, int heads, int dim, F f) {
    const int64_t t = k.dim() > 0 ? k.size(0) : 0;
    int64_t q_heads = 0, max_positions = 0, half = 0;
    pq_heads q_rows = {}, k_rows, v_rows;
    void *out = nullptr;
    if (o.q != Py_None) {
        const at::Tensor *q = tensor_of(o.q, "q");
        if (!q) return nullptr;
        q_heads = q->dim() == 3 ? q->size(1) : 0;
        if (q_heads > INT32_MAX) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
        if (!in_rows(o.q, type, {t, q_heads, dim}, "q", &q_rows) || !in_place(o.out, type, {t, q_heads, dim}, "out", &out)) return nullptr;
    }
    if ((o.cos == Py_None) != (o.sin == Py_None)) return PyErr_Format(PyExc_ValueError, "cos and sin go together");
    if (o.cos != Py_None) {
        const at::Tensor *cos = tensor_of(o.cos, "cos");
        if (!cos) return nullptr;
        if (cos->dim() != 2 || cos->size(1) > INT32_MAX / 2) return PyErr_Format(PyExc_ValueError, "cos and sin must be [positions][rot/2]");
        max_positions = cos->size(0);
        half = cos->size(1);
    }
    const int32_t *positions;
    const int64_t *slots;
    const float *cos_p, *sin_p, *q_weight, *k_weight;
    if (!in_rows(o.k, type, {t, heads, dim}, "k", &k_rows) || !in_rows(o.v, type, {t, heads, dim}, "v", &v_rows) ||
        !in_place(o.positions, at::kInt, {t}, "positions", &positions) || !in_place(o.slots, at::kLong, {t}, "slots", &slots) ||
        !in_place(o.cos, at::kFloat, {max_positions, half}, "cos", &cos_p, true) || !in_place(o.sin, at::kFloat, {max_positions, half}, "sin", &sin_p, true) ||
        !in_place(o.q_weight, at::kFloat, {dim}, "q_weight", &q_weight, true) || !in_place(o.k_weight, at::kFloat, {dim}, "k_weight", &k_weight, true))
        return nullptr;
    const double eps = PyFloat_AsDouble(o.eps);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    const int norm = PyObject_IsTrue(o.norm), pairs = PyObject_IsTrue(o.pairs);
    if (norm < 0 || pairs < 0) return nullptr;
    return without_gil([&] {
        return f(q_heads > 0 ? &q_rows : nullptr, (int)q_heads, &k_rows, &v_rows, t, positions, slots, cos_p, sin_p, max_positions, (int)(2 * half), pairs, norm,
                 q_weight, k_weight, (float)eps, out);
    });
}

// append(function, context, q, k, v, positions, slots, key_cache, value_cache, cos, sin, q_weight, k_weight, eps, norm, pairs, out)
PyObject *append(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 17) return PyErr_Format(PyExc_TypeError, "append takes 17 arguments");
    decltype(pq_kv_append) *f;
    pq_ctx *ctx;
    pq_kv_cache cache;
    if (!entry(args, &f, &ctx) || !read_cache(args[7], args[8], &cache)) return nullptr;
    const at::Tensor *k = tensor_of(args[3], "k");
    if (!k) return nullptr;
    const append_objects o = {args[2], args[3], args[4], args[5], args[6], args[9], args[10], args[11], args[12], args[13], args[14], args[15], args[16]};
    return append_rows(o, *k, THPVariable_Unpack(args[7]).scalar_type(), cache.heads, cache.dim, [&](auto... rest) { return f(ctx, &cache, rest...); });
}

// append8(function, context, q, k, v, positions, slots, key_cache, value_cache, key_scales, value_scales, cos, sin, q_weight, k_weight, eps,
//         norm, pairs, out): queries, keys and values of one type
PyObject *append8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 19) return PyErr_Format(PyExc_TypeError, "append8 takes 19 arguments");
    decltype(pq_kv_append8) *f;
    pq_ctx *ctx;
    pq_kv_cache8 cache;
    if (!entry(args, &f, &ctx) || !read_cache8(args[7], args[8], args[9], args[10], &cache)) return nullptr;
    const at::Tensor *k = tensor_of(args[3], "k");
    const int elem = k ? elem_of(*k, "k") : -1;
    if (elem < 0) return nullptr;
    const append_objects o = {args[2], args[3], args[4], args[5], args[6], args[11], args[12], args[13], args[14], args[15], args[16], args[17], args[18]};
    return append_rows(o, *k, k->scalar_type(), cache.heads, cache.dim, [&](auto... rest) { return f(ctx, &cache, (pq_elem)elem, rest...); });
}

// What attention and attention8 take alike; f: the library's function from the queries on.
struct attention_objects {
    PyObject *q, *block_tables, *cu_new, *kv_lens, *max_new, *scale, *window, *out, *lse;
};
template <class F> PyObject *attention_rows(const attention_objects &o, const at::Tensor &q, at::ScalarType type, int dim, F f) {
    int64_t max_new, window;
    if (!whole(o.max_new, &max_new) || !whole(o.window, &window)) return nullptr;
    const at::Tensor *tables = tensor_of(o.block_tables, "block_tables");
    if (!tables) return nullptr;
    if (tables->dim() != 2) return PyErr_Format(PyExc_ValueError, "block_tables must be [requests][width]");
    const int64_t t = q.dim() == 3 ? q.size(0) : 0, q_heads = q.dim() == 3 ? q.size(1) : 0, nreq = tables->size(0), width = tables->size(1);
    for (const int64_t x : {q_heads, nreq, width, max_new, window})
        if (x > INT32_MAX || x < INT32_MIN) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
    const double scale = o.scale == Py_None ? 1.0 / std::sqrt((double)dim) : PyFloat_AsDouble(o.scale);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    pq_heads q_rows;
    const int32_t *tables_p, *cu, *kv;
    void *out;
    float *lse;
    if (!in_rows(o.q, type, {t, q_heads, dim}, "q", &q_rows) || !in_place(o.block_tables, at::kInt, {nreq, width}, "block_tables", &tables_p) ||
        !in_place(o.cu_new, at::kInt, {nreq + 1}, "cu_new", &cu) || !in_place(o.kv_lens, at::kInt, {nreq}, "kv_lens", &kv) ||
        !in_place(o.out, type, {t, q_heads, dim}, "out", &out) || !in_place(o.lse, at::kFloat, {t, q_heads}, "lse", &lse))
        return nullptr;
    return without_gil([&] {
        return f(&q_rows, (int)q_heads, t, cu, kv, (int)nreq, tables_p, (int)width, (int)max_new, (float)scale, (int)window, out, lse);
    });
}

// attention(function, context, q, key_cache, value_cache, block_tables, cu_new, kv_lens, max_new, scale, window, out, lse)
PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 13) return PyErr_Format(PyExc_TypeError, "attention takes 13 arguments");
    decltype(pq_kv_attention) *f;
    pq_ctx *ctx;
    pq_kv_cache cache;
    if (!entry(args, &f, &ctx) || !read_cache(args[3], args[4], &cache)) return nullptr;
    const at::Tensor *q = tensor_of(args[2], "q");
    if (!q) return nullptr;
    const attention_objects o = {args[2], args[5], args[6], args[7], args[8], args[9], args[10], args[11], args[12]};
    return attention_rows(o, *q, THPVariable_Unpack(args[3]).scalar_type(), cache.dim, [&](auto... rest) { return f(ctx, &cache, rest...); });
}

// attention8(function, context, q, key_cache, value_cache, key_scales, value_scales, block_tables, cu_new, kv_lens, max_new, scale, window, out,
//            lse): queries and out of one type
PyObject *attention8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 15) return PyErr_Format(PyExc_TypeError, "attention8 takes 15 arguments");
    decltype(pq_kv_attention8) *f;
    pq_ctx *ctx;
    pq_kv_cache8 cache;
    if (!entry(args, &f, &ctx) || !read_cache8(args[3], args[4], args[5], args[6], &cache)) return nullptr;
    const at::Tensor *q = tensor_of(args[2], "q");
    const int elem = q ? elem_of(*q, "q") : -1;
    if (elem < 0) return nullptr;
    const attention_objects o = {args[2], args[7], args[8], args[9], args[10], args[11], args[12], args[13], args[14]};
    return attention_rows(o, *q, q->scalar_type(), cache.dim, [&](auto... rest) { return f(ctx, &cache, (pq_elem)elem, rest...); });
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

// logprobs(function, context, logits, tokens, top, logprobs, ranks, entropy, top_tokens, top_logprobs)
PyObject *logprobs(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 10) return PyErr_Format(PyExc_TypeError, "logprobs takes 10 arguments");
    decltype(pq_token_logprobs) *f;
    pq_ctx *ctx;
    int64_t top;
    if (!entry(args, &f, &ctx) || !whole(args[4], &top)) return nullptr;
    const at::Tensor *logits = tensor_of(args[2], "logits");
    if (!logits) return nullptr;
    const int elem = elem_of(*logits, "logits");
    if (elem < 0) return nullptr;
    if (logits->dim() != 2) return PyErr_Format(PyExc_ValueError, "logits must be [rows][vocab]");
    if (!rows_contiguous(*logits, "logits")) return nullptr;
    const int64_t rows = logits->size(0), vocab = logits->size(1);
    if (rows > INT32_MAX || vocab > INT32_MAX || top > INT32_MAX || top < INT32_MIN) return PyErr_Format(PyExc_ValueError, "sizes must be below 2^31");
    const int64_t *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *ranks;
    int64_t *top_tokens;
    // (a negative top is the library's to refuse)
    const int64_t listed = std::max<int64_t>(top, 0);
    if (!in_place(args[3], at::kLong, {rows}, "tokens", &tokens, true) || !in_place(args[5], at::kFloat, {rows}, "logprobs", &logprobs, true) ||
        !in_place(args[6], at::kInt, {rows}, "ranks", &ranks, true) || !in_place(args[7], at::kFloat, {rows}, "entropy", &entropy, true) ||
        !in_place(args[8], at::kLong, {rows, listed}, "top_tokens", &top_tokens, true) || !in_place(args[9], at::kFloat, {rows, listed}, "top_logprobs", &top_logprobs, true))
        return nullptr;
    const void *const p = logits->data_ptr();
    const int64_t row_stride = logits->stride(0);
    return without_gil([&] {
        return f(ctx, p, (pq_elem)elem, row_stride, (int)rows, (int)vocab, tokens, (int)top, logprobs, ranks, entropy, top_tokens, top_logprobs);
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
PyMethodDef methods[] = {METHOD(plan), METHOD(append), METHOD(attention), METHOD(sample), METHOD(append8), METHOD(attention8), METHOD(logprobs), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tensor_views", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_tensor_views(void) { return PyModule_Create(&module); }
