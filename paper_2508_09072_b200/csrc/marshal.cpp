// Argument marshalling of the prompt calls (reader_prompt_append, reader_tree_rotate, reader_prompt_attn), of the 4-bit cache
// (reader_q4_*) and of the page calls (reader_pages_*) for Python:
// a CPython extension module that checks torch tensors and calls the C ABI with their addresses.  It does what the
// ctypes code of binding.py does for the other calls; it is native because these calls are as short as 4 to 10 us on
// the GPU, and looking at a dozen tensors from Python took 8 to 12 us of the host's time (here: below 2 us).
//
// The functions return (status code of the library, outputs ...); binding.py turns a code into its exception.  A
// wrong tensor raises TypeError (type, layout) or ValueError (shape, device) before anything is called.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>
#include <vector>

#include "reader_verify.h"

namespace {

struct Wrong {
    PyObject *type;
    std::string text;
};
[[noreturn]] void wrong_type(const char *name, const char *what) { throw Wrong{PyExc_TypeError, std::string(name) + ": " + what}; }
[[noreturn]] void wrong_value(const char *name, const char *what) { throw Wrong{PyExc_ValueError, std::string(name) + ": " + what}; }

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) wrong_type(name, "need a tensor");
    return THPVariable_Unpack(o);
}

void here(const at::Tensor &t, int device, const char *name) {
    if (!t.is_cuda()) wrong_type(name, "need a CUDA tensor");
    if (t.get_device() != device) wrong_value(name, "is on another device than this reader");
}

// A contiguous tensor of that type on the reader's device.
const at::Tensor &dense(PyObject *o, at::ScalarType type, int dim, int device, const char *name) {
    const at::Tensor &t = tensor(o, name);
    here(t, device, name);
    if (t.scalar_type() != type) wrong_type(name, (std::string("need dtype ") + c10::toString(type)).c_str());
    if (!t.is_contiguous()) wrong_type(name, "need a contiguous tensor");
    if (t.dim() != dim) wrong_value(name, "has another number of dimensions");
    return t;
}
void *address(const at::Tensor &t) { return t.data_ptr(); }

// A bf16 tensor [..., heads, head_dim] whose heads are dense and whose tokens are evenly spaced (a tensor of its own or a
// part of a fused projection's output); its token stride in elements.
struct Heads {
    const at::Tensor *t;
    int64_t stride;
};
Heads heads_of(PyObject *o, int dim, int device, const char *name) {
    const at::Tensor &t = tensor(o, name);
    here(t, device, name);
    if (t.scalar_type() != at::kBFloat16) wrong_type(name, "need dtype BFloat16");
    if (t.dim() != dim) wrong_value(name, "has another number of dimensions");
    const int64_t heads = t.size(dim - 2), d = t.size(dim - 1);
    if (t.numel() == 0) return {&t, heads * d};
    if ((d > 1 && t.stride(dim - 1) != 1) || (heads > 1 && t.stride(dim - 2) != d)) wrong_value(name, "the heads of a token must be dense");
    if (dim == 3) return {&t, t.size(0) > 1 ? t.stride(0) : heads * d};
    const int64_t b = t.size(0), n = t.size(1);
    if (b > 1 && n > 1 && t.stride(0) != n * t.stride(1)) wrong_value(name, "the tokens must be evenly spaced");
    return {&t, n > 1 ? t.stride(1) : b > 1 ? t.stride(0) : heads * d};
}

int32_t small(int64_t x, const char *name) {
    if (x < 0 || x > INT32_MAX) wrong_value(name, "is too large");
    return (int32_t)x;
}
int64_t integer(PyObject *o, const char *name) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        wrong_type(name, "need an integer");
    }
    return x;
}
float real(PyObject *o, const char *name) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        wrong_type(name, "need a number");
    }
    return (float)x;
}

bool truth(PyObject *o, const char *name) {
    const int x = PyObject_IsTrue(o);
    if (x < 0) {
        PyErr_Clear();
        wrong_type(name, "need a truth value");
    }
    return x != 0;
}

struct Cache {
    reader_kv_cache c;
    int32_t batch;
};
// args: k_pool, v_pool, page_table, seq_lens, shared_prefix_len
Cache cache_of(PyObject *const *a, int device) {
    const at::Tensor &k = dense(a[0], at::kBFloat16, 4, device, "k_pool"), &v = dense(a[1], at::kBFloat16, 4, device, "v_pool");
    const at::Tensor &table = dense(a[2], at::kInt, 2, device, "page_table"), &lens = dense(a[3], at::kInt, 1, device, "seq_lens");
    if (v.sizes() != k.sizes()) wrong_value("v_pool", "need the shape of k_pool");
    if (lens.size(0) != table.size(0)) wrong_value("seq_lens", "need one length for each row of the page table");
    Cache r;
    r.batch = small(table.size(0), "page_table");
    r.c.k_pool = address(k);
    r.c.v_pool = address(v);
    r.c.num_pages = small(k.size(0), "k_pool");
    r.c.page_size = small(k.size(2), "k_pool");
    r.c.n_kv_heads = small(k.size(1), "k_pool");
    r.c.head_dim = small(k.size(3), "k_pool");
    r.c.page_table = static_cast<const int32_t *>(address(table));
    r.c.max_pages_per_seq = small(table.size(1), "page_table");
    r.c.seq_lens = static_cast<int32_t *>(address(lens));
    r.c.shared_prefix_len = small(integer(a[4], "shared_prefix_len"), "shared_prefix_len");
    return r;
}

// args: rope, q_weight, k_weight, eps, interleaved
reader_rotation rotation_of(PyObject *const *a, int64_t head_dim, int device) {
    reader_rotation r{};
    if (a[0] != Py_None) {
        const at::Tensor &rope = dense(a[0], at::kFloat, 3, device, "rope");
        if (rope.size(1) != 2) wrong_value("rope", "need [max_positions, 2, rot_dim / 2]");
        r.rope = static_cast<const float *>(address(rope));
        r.max_positions = small(rope.size(0), "rope");
        r.rot_dim = small(2 * rope.size(2), "rope");
    }
    for (int i = 1; i < 3; ++i) {
        if (a[i] == Py_None) continue;
        const char *name = i == 1 ? "q_weight" : "k_weight";
        const at::Tensor &w = dense(a[i], at::kBFloat16, 1, device, name);
        if (w.size(0) != head_dim) wrong_value(name, "need one weight for each element of a head");
        (i == 1 ? r.q_weight : r.k_weight) = address(w);
    }
    r.eps = real(a[3], "eps");
    r.interleaved = truth(a[4], "interleaved");
    return r;
}

reader_prompt prompt_of(PyObject *o, int32_t batch, int64_t tokens, int device) {
    const at::Tensor &start = dense(o, at::kInt, 1, device, "token_start");
    if (start.size(0) != (int64_t)batch + 1) wrong_value("token_start", "need one entry more than the cache has sequences");
    return {batch, small(tokens, "q"), static_cast<const int32_t *>(address(start))};
}

// An output: what the caller gave, of the right shape, or a new tensor.
at::Tensor output(PyObject *o, at::IntArrayRef shape, at::ScalarType type, int device, const char *name) {
    if (o == Py_None) return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, device));
    const at::Tensor &t = dense(o, type, (int)shape.size(), device, name);
    if (t.sizes() != shape) wrong_value(name, "has another shape");
    return t;
}
PyObject *given_back(PyObject *o, const at::Tensor &t) {
    if (o == Py_None) return THPVariable_Wrap(t);
    Py_INCREF(o);
    return o;
}
// A new tuple of the code and references that are handed over.
template <size_t N>
PyObject *results(reader_status st, PyObject *const (&o)[N]) {
    PyObject *t = PyTuple_New(1 + N);
    PyObject *code = PyLong_FromLong(st);
    bool ok = t && code;
    for (PyObject *x : o) ok = ok && x;
    if (!ok) {
        Py_XDECREF(t);
        Py_XDECREF(code);
        for (PyObject *x : o) Py_XDECREF(x);
        return nullptr;
    }
    PyTuple_SET_ITEM(t, 0, code);
    for (size_t i = 0; i < N; ++i) PyTuple_SET_ITEM(t, 1 + i, o[i]);
    return t;
}

// The current device's current stream, as for every other call (the library refuses a device that is not its context's).
void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

reader_ctx *context(PyObject *o) { return reinterpret_cast<reader_ctx *>((uintptr_t)integer(o, "handle")); }

template <typename F>
PyObject *guarded(const char *name, Py_ssize_t have, Py_ssize_t want, const F &f) {
    if (have != want) {
        PyErr_Format(PyExc_TypeError, "%s: %zd arguments, %zd wanted", name, have, want);
        return nullptr;
    }
    try {
        return f();
    } catch (const Wrong &w) {
        PyErr_SetString(w.type, w.text.c_str());
    } catch (const std::exception &e) {   // (out of memory in an output's allocation, for one)
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// handle, device, q, k, v, (cache: 5), token_start, (rotation: 5), out, status
PyObject *prompt_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("prompt_append", n, 18, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        Cache c = cache_of(a + 5, device);
        const Heads q = heads_of(a[2], 3, device, "q"), k = heads_of(a[3], 3, device, "k"), v = heads_of(a[4], 3, device, "v");
        const int64_t tokens = q.t->size(0), hq = q.t->size(1), d = q.t->size(2), kv[3] = {tokens, c.c.n_kv_heads, c.c.head_dim};
        if (d != c.c.head_dim) wrong_value("q", "its head dimension is not the cache's");
        if (k.t->sizes() != at::IntArrayRef(kv, 3)) wrong_value("k", "need [tokens, KV heads, head_dim]");
        if (v.t->sizes() != at::IntArrayRef(kv, 3)) wrong_value("v", "need [tokens, KV heads, head_dim]");
        const reader_prompt p = prompt_of(a[10], c.batch, tokens, device);
        const reader_rotation r = rotation_of(a + 11, d, device);
        const at::Tensor out = output(a[16], q.t->sizes(), at::kBFloat16, device, "out");
        const at::Tensor status = output(a[17], {c.batch}, at::kInt, device, "status");
        const reader_status st =
            reader_prompt_append(context(a[0]), address(*q.t), address(*k.t), address(*v.t), q.stride, k.stride, v.stride, small(hq, "q"), &c.c,
                                 &p, &r, address(out), static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[16], out), given_back(a[17], status)});
    });
}

// handle, device, q, k, v, seq_lens, parent, (rotation: 5), out, k_tree, v_tree, status
PyObject *tree_rotate(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("tree_rotate", n, 16, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        const Heads q = heads_of(a[2], 4, device, "q"), k = heads_of(a[3], 4, device, "k"), v = heads_of(a[4], 4, device, "v");
        const int64_t B = q.t->size(0), T = q.t->size(1), d = q.t->size(3), hkv = k.t->size(2), kv[4] = {B, T, hkv, d};
        if (k.t->sizes() != at::IntArrayRef(kv, 4)) wrong_value("k", "need [batch, nodes, KV heads, head_dim]");
        if (v.t->sizes() != at::IntArrayRef(kv, 4)) wrong_value("v", "need [batch, nodes, KV heads, head_dim]");
        const at::Tensor &lens = dense(a[5], at::kInt, 1, device, "seq_lens"), &parent = dense(a[6], at::kInt, 2, device, "parent");
        if (parent.size(0) != B || parent.size(1) != T) wrong_value("parent", "need [batch, nodes]");
        if (lens.size(0) != B) wrong_value("seq_lens", "need one length for each sequence");
        const reader_rotation r = rotation_of(a + 7, d, device);
        const reader_tree tree = {small(B, "q"), small(T, "q"), static_cast<const int32_t *>(address(parent)), nullptr};
        const at::Tensor out = output(a[12], q.t->sizes(), at::kBFloat16, device, "out");
        const at::Tensor k_tree = output(a[13], k.t->sizes(), at::kBFloat16, device, "k_tree");
        const at::Tensor v_tree = output(a[14], v.t->sizes(), at::kBFloat16, device, "v_tree");
        const at::Tensor status = output(a[15], {B}, at::kInt, device, "status");
        const reader_status st = reader_tree_rotate(
            context(a[0]), address(*q.t), address(*k.t), address(*v.t), q.stride, k.stride, v.stride, small(q.t->size(2), "q"), small(hkv, "k"),
            small(d, "q"), &tree, static_cast<const int32_t *>(address(lens)), &r, address(out), address(k_tree), address(v_tree),
            static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[12], out), given_back(a[13], k_tree), given_back(a[14], v_tree), given_back(a[15], status)});
    });
}

// handle, device, q, (cache: 5), token_start, scale, update_seq_lens, out, lse, workspace, status
PyObject *prompt_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("prompt_attn", n, 15, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        Cache c = cache_of(a + 3, device);
        const at::Tensor &q = dense(a[2], at::kBFloat16, 3, device, "q");
        const int64_t tokens = q.size(0), hq = q.size(1);
        if (q.size(2) != c.c.head_dim) wrong_value("q", "its head dimension is not the cache's");
        const reader_prompt p = prompt_of(a[8], c.batch, tokens, device);
        const float scale = real(a[9], "scale");
        const bool update = truth(a[10], "update_seq_lens");
        const at::Tensor out = output(a[11], q.sizes(), at::kBFloat16, device, "out");
        float *lse = nullptr;
        if (a[12] != Py_None) {
            const at::Tensor &t = dense(a[12], at::kFloat, 2, device, "lse");
            if (t.size(0) != tokens || t.size(1) != hq) wrong_value("lse", "need [tokens, heads]");
            lse = static_cast<float *>(address(t));
        }
        const at::Tensor &ws = dense(a[13], at::kByte, 1, device, "workspace");
        const at::Tensor status = output(a[14], {c.batch}, at::kInt, device, "status");
        const reader_status st = reader_prompt_attn(context(a[0]), address(q), small(hq, "q"), &c.c, &p, scale, update,
                                                    address(out), lse, address(ws), (size_t)ws.numel(),
                                                    static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[11], out), given_back(a[14], status)});
    });
}

// ---- the 4-bit cache and the page calls

// A name that attributes are asked for by, made once (a string made for every question costs more than the question).
struct Name {
    const char *text;
    PyObject *o;
    explicit Name(const char *s) : text(s), o(PyUnicode_InternFromString(s)) {}
};
// An attribute of a cache or pages object, for as long as this lives.
struct Attr {
    PyObject *o;
    Attr(PyObject *from, const Name &name) : o(name.o ? PyObject_GetAttr(from, name.o) : nullptr) {
        if (!o) {
            PyErr_Clear();
            wrong_type(name.text, "the object has no such attribute");
        }
    }
    ~Attr() { Py_DECREF(o); }
    Attr(const Attr &) = delete;
};
// The items of a list or tuple.
struct Items {
    PyObject *seq;
    Py_ssize_t n;
    Items(PyObject *o, const char *name) : seq(PySequence_Fast(o, "")), n(0) {
        if (!seq) {
            PyErr_Clear();
            wrong_type(name, "need a list");
        }
        n = PySequence_Fast_GET_SIZE(seq);
    }
    ~Items() { Py_DECREF(seq); }
    Items(const Items &) = delete;
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(seq, i); }
};

const Name &k_pool_name() { static const Name n("k_pool"); return n; }
const Name &v_pool_name() { static const Name n("v_pool"); return n; }
const Name &table_name() { static const Name n("page_table"); return n; }
const Name &lens_name() { static const Name n("seq_lens"); return n; }
const Name &prefix_name() { static const Name n("shared_prefix_len"); return n; }
const Name &refs_name() { static const Name n("refs"); return n; }
const Name &pools_name() { static const Name n("pools"); return n; }

// A KvCache (bf16 pools) or a Q4Cache (4-bit ones).
Cache cache_object(PyObject *o, bool narrow, int device) {
    const Attr ko(o, k_pool_name()), vo(o, v_pool_name()), to(o, table_name()), lo(o, lens_name()), po(o, prefix_name());
    if (!narrow) {
        PyObject *const a[5] = {ko.o, vo.o, to.o, lo.o, po.o};
        return cache_of(a, device);
    }
    const at::Tensor &k = dense(ko.o, at::kByte, 3, device, "k_pool"), &v = dense(vo.o, at::kByte, 3, device, "v_pool");
    const at::Tensor &table = dense(to.o, at::kInt, 2, device, "page_table"), &lens = dense(lo.o, at::kInt, 1, device, "seq_lens");
    if (v.sizes() != k.sizes()) wrong_value("v_pool", "need the shape of k_pool");
    if (lens.size(0) != table.size(0)) wrong_value("seq_lens", "need one length for each row of the page table");
    if (k.size(2) % 36 != 0) wrong_value("k_pool", "need [num_pages, KV heads, 36 * head_dim]");
    Cache r;
    r.batch = small(table.size(0), "page_table");
    r.c.k_pool = address(k);
    r.c.v_pool = address(v);
    r.c.num_pages = small(k.size(0), "k_pool");
    r.c.page_size = READER_PAGE_SIZE;
    r.c.n_kv_heads = small(k.size(1), "k_pool");
    r.c.head_dim = small(k.size(2) / 36, "k_pool");
    r.c.page_table = static_cast<const int32_t *>(address(table));
    r.c.max_pages_per_seq = small(table.size(1), "page_table");
    r.c.seq_lens = static_cast<int32_t *>(address(lens));
    r.c.shared_prefix_len = small(integer(po.o, "shared_prefix_len"), "shared_prefix_len");
    return r;
}
std::vector<reader_kv_cache> cache_list(PyObject *o, bool narrow, int device, int32_t batch, const char *name) {
    const Items items(o, name);
    if (items.n == 0) wrong_value(name, "need one cache at least");
    std::vector<reader_kv_cache> r;
    r.reserve(items.n);
    for (Py_ssize_t i = 0; i < items.n; ++i) {
        const Cache c = cache_object(items[i], narrow, device);
        if (c.batch != batch) wrong_value(name, "its page table has another number of rows");
        r.push_back(c.c);
    }
    return r;
}
const int32_t *ints(PyObject *o, int64_t n, int device, const char *name) {
    const at::Tensor &t = dense(o, at::kInt, 1, device, name);
    if (t.size(0) != n) wrong_value(name, "has another number of entries");
    return static_cast<const int32_t *>(address(t));
}

// handle, device, store, from, to, first, last, status
PyObject *q4_convert(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("q4_convert", n, 8, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        const bool store = truth(a[2], "store");
        const int32_t batch = small(dense(a[5], at::kInt, 1, device, "first").size(0), "first");
        const int32_t *first = ints(a[5], batch, device, "first"), *last = ints(a[6], batch, device, "last");
        const std::vector<reader_kv_cache> from = cache_list(a[3], !store, device, batch, "source"), to = cache_list(a[4], store, device, batch, "destination");
        if (from.size() != to.size()) wrong_value("destination", "need one cache for each of the source's");
        const at::Tensor status = output(a[7], {batch}, at::kInt, device, "status");
        const reader_status st = (store ? reader_q4_store : reader_q4_load)(context(a[0]), from.data(), to.data(), (int32_t)from.size(), batch, first, last,
                                                                           static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[7], status)});
    });
}

// handle, device, caches, k_trees, v_trees, path, n_acc, update_seq_lens, slots, status
PyObject *q4_commit(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("q4_commit", n, 10, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        const at::Tensor &path = dense(a[5], at::kInt, 2, device, "path");
        const int64_t B = path.size(0), max_path = path.size(1);
        const int32_t *n_acc = ints(a[6], B, device, "n_acc");
        const std::vector<reader_kv_cache> caches = cache_list(a[2], true, device, small(B, "path"), "caches");
        const Items k(a[3], "k_trees"), v(a[4], "v_trees");
        if (k.n != (Py_ssize_t)caches.size() || v.n != k.n) wrong_value("k_trees", "need a tensor of keys and one of values for each cache");
        std::vector<const void *> kp, vp;
        int64_t nodes = 0;
        for (Py_ssize_t i = 0; i < k.n; ++i) {
            const at::Tensor &x = dense(k[i], at::kBFloat16, 4, device, "k_trees"), &y = dense(v[i], at::kBFloat16, 4, device, "v_trees");
            if (i == 0) nodes = x.size(1);
            const int64_t want[4] = {B, nodes, caches[i].n_kv_heads, caches[i].head_dim};
            if (x.sizes() != at::IntArrayRef(want, 4)) wrong_value("k_trees", "need [batch, nodes, KV heads, head_dim]");
            if (y.sizes() != at::IntArrayRef(want, 4)) wrong_value("v_trees", "need [batch, nodes, KV heads, head_dim]");
            kp.push_back(address(x));
            vp.push_back(address(y));
        }
        const bool update = truth(a[7], "update_seq_lens");
        const at::Tensor slots = output(a[8], path.sizes(), at::kInt, device, "slots"), status = output(a[9], {B}, at::kInt, device, "status");
        const reader_status st = reader_q4_commit(context(a[0]), caches.data(), kp.data(), vp.data(), (int32_t)caches.size(), small(B, "path"),
                                                  small(nodes, "k_trees"), static_cast<const int32_t *>(address(path)), n_acc, small(max_path, "path"), update,
                                                  static_cast<int32_t *>(address(slots)), static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[8], slots), given_back(a[9], status)});
    });
}

// handle, device, q, k_tree, v_tree, cache, parent, scale, anc_mask, out, lse, status, workspace
PyObject *q4_verify_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("q4_verify_attn", n, 13, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        const Cache c = cache_object(a[5], true, device);
        const at::Tensor &q = dense(a[2], at::kBFloat16, 4, device, "q"), &k = dense(a[3], at::kBFloat16, 4, device, "k_tree"),
                         &v = dense(a[4], at::kBFloat16, 4, device, "v_tree"), &parent = dense(a[6], at::kInt, 2, device, "parent");
        const int64_t B = q.size(0), T = q.size(1), hq = q.size(2), kv[4] = {B, T, c.c.n_kv_heads, c.c.head_dim};
        if (B != c.batch) wrong_value("q", "need one tree for each row of the page table");
        if (q.size(3) != c.c.head_dim) wrong_value("q", "its head dimension is not the cache's");
        if (k.sizes() != at::IntArrayRef(kv, 4)) wrong_value("k_tree", "need [batch, nodes, KV heads, head_dim]");
        if (v.sizes() != at::IntArrayRef(kv, 4)) wrong_value("v_tree", "need [batch, nodes, KV heads, head_dim]");
        if (parent.size(0) != B || parent.size(1) != T) wrong_value("parent", "need [batch, nodes]");
        reader_tree tree = {small(B, "q"), small(T, "q"), static_cast<const int32_t *>(address(parent)), nullptr};
        if (a[8] != Py_None) {
            const at::Tensor &anc = dense(a[8], at::kLong, 3, device, "anc_mask");
            if (anc.size(0) != B || anc.size(1) != T || anc.size(2) != 2) wrong_value("anc_mask", "need [batch, nodes, 2]");
            tree.anc_mask = static_cast<const uint64_t *>(address(anc));
        }
        const float scale = real(a[7], "scale");
        const at::Tensor out = output(a[9], q.sizes(), at::kBFloat16, device, "out");
        float *lse = nullptr;
        if (a[10] != Py_None) {
            const at::Tensor &t = dense(a[10], at::kFloat, 3, device, "lse");
            if (t.size(0) != B || t.size(1) != T || t.size(2) != hq) wrong_value("lse", "need [batch, nodes, heads]");
            lse = static_cast<float *>(address(t));
        }
        const at::Tensor status = output(a[11], {B}, at::kInt, device, "status");
        const at::Tensor &ws = dense(a[12], at::kByte, 1, device, "workspace");
        const reader_status st = reader_q4_verify_attn(context(a[0]), address(q), small(hq, "q"), address(k), address(v), &c.c, &tree, scale, address(out), lse,
                                                       address(ws), (size_t)ws.numel(), static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[9], out), given_back(a[11], status)});
    });
}

struct PagesArgs {
    reader_pages p;
    std::vector<void *> pools;
};
int64_t bytes_of_page(const at::Tensor &t, int64_t num_pages, const char *name) {
    if (!t.is_contiguous()) wrong_type(name, "need contiguous tensors");
    if (t.dim() < 1 || t.size(0) != num_pages) wrong_value(name, "need one page for each of the counts");
    return num_pages ? (int64_t)t.nbytes() / num_pages : 0;
}
void pages_of(PyObject *o, int device, bool with_pools, PagesArgs &r) {
    const Attr ro(o, refs_name()), to(o, table_name()), lo(o, lens_name());
    const at::Tensor &refs = dense(ro.o, at::kInt, 1, device, "refs"), &table = dense(to.o, at::kInt, 2, device, "page_table");
    r.p = reader_pages{};
    r.p.refs = static_cast<int32_t *>(address(refs));
    r.p.num_pages = small(refs.size(0), "refs");
    r.p.page_table = static_cast<int32_t *>(address(table));
    r.p.rows = small(table.size(0), "page_table");
    r.p.max_pages_per_seq = small(table.size(1), "page_table");
    r.p.seq_lens = const_cast<int32_t *>(ints(lo.o, table.size(0), device, "seq_lens"));
    if (!with_pools) return;
    const Attr po(o, pools_name());
    const Items pools(po.o, "pools");
    for (Py_ssize_t i = 0; i < pools.n; ++i) {
        const at::Tensor &t = tensor(pools[i], "pools");
        here(t, device, "pools");
        const int64_t bytes = bytes_of_page(t, refs.size(0), "pools");
        if (i > 0 && (size_t)bytes != r.p.page_bytes) wrong_value("pools", "need pages of one size");
        r.p.page_bytes = (size_t)bytes;
        r.pools.push_back(address(t));
    }
    r.p.pools = r.pools.data();
    r.p.n_pools = small(pools.n, "pools");
}

// handle, device, pages, src, dst, workspace, status (fork) / handle, device, pages, rows, tokens, workspace, status (reserve)
template <bool kFork>
PyObject *pages_requests(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(kFork ? "pages_fork" : "pages_reserve", n, 7, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        PagesArgs p;
        pages_of(a[2], device, !kFork, p);
        const char *name = kFork ? "src" : "rows";
        const int32_t count = small(dense(a[3], at::kInt, 1, device, name).size(0), name);
        const int32_t *x = ints(a[3], count, device, name), *y = ints(a[4], count, device, kFork ? "dst" : "tokens");
        const at::Tensor &ws = dense(a[5], at::kByte, 1, device, "workspace");
        const at::Tensor status = output(a[6], {count}, at::kInt, device, "status");
        const reader_status st = (kFork ? reader_pages_fork : reader_pages_reserve)(context(a[0]), &p.p, x, y, count, address(ws), (size_t)ws.numel(),
                                                                                   static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[6], status)});
    });
}

// handle, device, pages, rows, keep, status
PyObject *pages_free(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("pages_free", n, 6, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        PagesArgs p;
        pages_of(a[2], device, false, p);
        const int32_t count = small(dense(a[3], at::kInt, 1, device, "rows").size(0), "rows");
        const int32_t *rows = ints(a[3], count, device, "rows"), *keep = a[4] == Py_None ? nullptr : ints(a[4], count, device, "keep");
        const at::Tensor status = output(a[5], {count}, at::kInt, device, "status");
        const reader_status st = reader_pages_free(context(a[0]), &p.p, rows, keep, count, static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[5], status)});
    });
}

// handle, device, pages, workspace, n_used[, new_ids]
PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("pages_compact", n == 6 ? 5 : n, 5, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        PagesArgs p;
        pages_of(a[2], device, true, p);
        const at::Tensor &ws = dense(a[3], at::kByte, 1, device, "workspace");
        const at::Tensor used = output(a[4], {1}, at::kInt, device, "n_used");
        int32_t *new_ids = n == 6 && a[5] != Py_None ? const_cast<int32_t *>(ints(a[5], p.p.num_pages, device, "new_ids")) : nullptr;
        const reader_status st =
            reader_pages_compact_map(context(a[0]), &p.p, static_cast<int32_t *>(address(used)), new_ids, address(ws), (size_t)ws.numel(), stream());
        return results(st, {given_back(a[4], used)});
    });
}

// handle, device, from_pools, to_pools, from_ids, to_ids, status
PyObject *pages_copy(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded("pages_copy", n, 7, [&]() -> PyObject * {
        const int device = (int)integer(a[1], "device");
        const Items from(a[2], "from_pools"), to(a[3], "to_pools");
        if (from.n == 0 || from.n != to.n) wrong_value("to_pools", "need one pool for each of from_pools, and one at least");
        std::vector<const void *> fp;
        std::vector<void *> tp;
        int64_t from_pages = 0, to_pages = 0, bytes = 0;
        for (Py_ssize_t i = 0; i < from.n; ++i) {
            const at::Tensor &x = tensor(from[i], "from_pools"), &y = tensor(to[i], "to_pools");
            here(x, device, "from_pools");
            here(y, device, "to_pools");
            if (i == 0 && (x.dim() < 1 || y.dim() < 1 || x.size(0) < 1 || y.size(0) < 1)) wrong_value("from_pools", "need one page at least");
            if (i == 0) { from_pages = x.size(0); to_pages = y.size(0); }
            const int64_t b = bytes_of_page(x, from_pages, "from_pools");
            if (i == 0) bytes = b;
            if (b != bytes || bytes_of_page(y, to_pages, "to_pools") != bytes) wrong_value("to_pools", "need pages of one size");
            fp.push_back(address(x));
            tp.push_back(address(y));
        }
        const int32_t count = small(dense(a[4], at::kInt, 1, device, "from_ids").size(0), "from_ids");
        const int32_t *x = ints(a[4], count, device, "from_ids"), *y = ints(a[5], count, device, "to_ids");
        const at::Tensor status = output(a[6], {count}, at::kInt, device, "status");
        const reader_status st = reader_pages_copy(context(a[0]), fp.data(), small(from_pages, "from_pools"), tp.data(), small(to_pages, "to_pools"),
                                                   small(from.n, "from_pools"), (size_t)bytes, x, y, count, static_cast<int32_t *>(address(status)), stream());
        return results(st, {given_back(a[6], status)});
    });
}

#define METHOD(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    METHOD("q4_convert", q4_convert),
    METHOD("q4_commit", q4_commit),
    METHOD("q4_verify_attn", q4_verify_attn),
    METHOD("pages_fork", pages_requests<true>),
    METHOD("pages_reserve", pages_requests<false>),
    METHOD("pages_free", pages_free),
    METHOD("pages_compact", pages_compact),
    METHOD("pages_copy", pages_copy),
    {"prompt_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(prompt_append)), METH_FASTCALL, nullptr},
    {"tree_rotate", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(tree_rotate)), METH_FASTCALL, nullptr},
    {"prompt_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(prompt_attn)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
