// What DsfqLinear does on the host between two launches, in native code: the checks of a call's tensors, the output's allocation, the current
// stream, the call of the C entry point with the interpreter's lock released.  The same as the Python functions of binding.py do one by one
// (a call of two launches, 64 x 128 -> 128 in f32 when it was one: 11.5 us with them, 8.9 this way, of which 7.2 are the launches).
//
// linear(kind, X, signs, inv_smooth, gelu_table, W, w_scale, bias, out, workspace, N, bits)
//   -> the output, or the entry point's status where it is not 0, or NotImplemented, before anything is launched, where a call is not an ordinary
//      one: an argument that is no plain contiguous GPU tensor (a subclass, a wrapper, a view that is not contiguous), an X that is not
//      two-dimensional bf16 or f32, an output that cannot be allocated.  The caller's Python path takes it then, with its errors.  As there, types
//      of the other operands and which GPU holds what are the caller's to get right.
// bind(kind, address): the C entry point of a kind.
//
// kv4_append(K, V, signs, slots, cache, page_tokens, rope, positions, rope_pair), kv4_read(cache, page_tokens, signs, slots, K, V) and kv4_attention(Q, signs, scale, causal, cache,
// page_tokens, kv_heads, page_table, q_starts, kv_lens, max_q, max_kv, out, workspace, rope, positions, rope_pair): the calls of binding.py's functions of these names, on the current
// stream (a token appended and read back 17 us with those, 9 this way)
//   -> the entry point's status, or NotImplemented, before anything is launched, where a call is not an ordinary one (an argument of another type, shape or kind than those
//      functions take): they refuse it, or take it, then.
// bind_kv4(which, address): their C entry points, in this order.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <cstdint>

namespace {

enum Kind { kPacked, kE2m3, kGelu, kInt8, kInt8Blocks, kKinds };
void *entry[kKinds];

using PackedFn = int (*)(const void *, int, int, int, int, const void *, const void *, const void *, const void *, const void *, void *, void *, size_t, void *);
using GeluFn = int (*)(const void *, int, int, int, int, const void *, const void *, const void *, const void *, const void *, const void *, void *, void *, size_t, void *);
using Int8Fn = int (*)(const void *, int, int, int, int, const void *, const void *, int, const void *, const void *, const void *, void *, void *, size_t, void *);

// the tensor behind an argument, if it is an ordinary one on the GPU, contiguous and with memory of its own kind; nullptr otherwise
const at::Tensor *ordinary(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.has_storage() || !t.is_cuda() || !t.is_contiguous() || t.is_conj() || t.is_neg()) return nullptr;
    return &t;
}

// device address of a tensor, or nullptr for None; false if the argument is neither
bool address(PyObject *o, const void **p)
{
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = ordinary(o);
    if (t == nullptr) return false;
    *p = t->const_data_ptr();
    return true;
}

PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 12) {
        PyErr_SetString(PyExc_TypeError, "linear takes 12 arguments");
        return nullptr;
    }
    bool launched = false;
    try {
        const long kind = PyLong_AsLong(args[0]), N_layer = PyLong_AsLong(args[10]), bits = PyLong_AsLong(args[11]);
        if (PyErr_Occurred()) return nullptr;
        if (kind < 0 || kind >= kKinds || entry[kind] == nullptr) Py_RETURN_NOTIMPLEMENTED;
        const at::Tensor *X = ordinary(args[1]), *ws = ordinary(args[9]);
        if (X == nullptr || ws == nullptr || X->dim() != 2 || X->size(0) > INT32_MAX || X->size(1) > INT32_MAX) Py_RETURN_NOTIMPLEMENTED;
        const at::ScalarType type = X->scalar_type();
        if (type != at::kBFloat16 && type != at::kFloat) Py_RETURN_NOTIMPLEMENTED;
        const void *signs, *inv, *table, *W, *w_scale, *bias;
        if (!address(args[2], &signs) || !address(args[3], &inv) || !address(args[4], &table) || !address(args[5], &W) || !address(args[6], &w_scale) ||
            !address(args[7], &bias))
            Py_RETURN_NOTIMPLEMENTED;
        const int M = (int)X->size(0), K = (int)X->size(1);
        at::Tensor made;
        const at::Tensor *Y = nullptr;
        if (args[8] == Py_None) {
            made = at::empty({M, N_layer}, X->options().dtype(at::kBFloat16));
            Y = &made;
        } else {
            Y = ordinary(args[8]);
            if (Y == nullptr || Y->dim() != 2 || Y->size(1) > INT32_MAX) Py_RETURN_NOTIMPLEMENTED;
        }
        const int N = (int)Y->size(1);
        const void *x = X->const_data_ptr();
        void *y = Y->data_ptr(), *w = ws->data_ptr();
        const size_t w_bytes = (size_t)ws->numel() * ws->element_size();
        const int dtype = type == at::kFloat;                       // QVGGT_BF16 = 0, QVGGT_F32 = 1
        void *stream = reinterpret_cast<void *>(c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream());
        int status;
        launched = true;
        Py_BEGIN_ALLOW_THREADS
        switch (kind) {
            case kGelu: status = reinterpret_cast<GeluFn>(entry[kind])(x, dtype, M, N, K, signs, inv, table, W, w_scale, bias, y, w, w_bytes, stream); break;
            case kInt8:
            case kInt8Blocks: status = reinterpret_cast<Int8Fn>(entry[kind])(x, dtype, M, N, K, signs, inv, (int)bits, W, w_scale, bias, y, w, w_bytes, stream); break;
            default: status = reinterpret_cast<PackedFn>(entry[kind])(x, dtype, M, N, K, signs, inv, W, w_scale, bias, y, w, w_bytes, stream); break;
        }
        Py_END_ALLOW_THREADS
        if (status != 0) return PyLong_FromLong(status);
        if (args[8] == Py_None) return THPVariable_Wrap(std::move(made));
        Py_INCREF(args[8]);
        return args[8];
    } catch (python_error &e) {                                     // raised in Python: a dispatch mode that sees the allocation
        e.restore();
        return nullptr;
    } catch (const std::exception &e) {
        if (!launched) Py_RETURN_NOTIMPLEMENTED;                    // torch's own errors, the allocator's among them: torch.empty raises them as Python knows them
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// ---- the 4-bit key/value cache
enum { kAppend, kRead, kAttention, kKv4 };
void *kv4_entry[kKv4];
using AppendFn = int (*)(const void *, const void *, int, int, long long, long long, int, int, const void *, int, int, int, const void *, const void *, const void *, void *, int, int, void *);
using ReadFn = int (*)(const void *, int, int, int, int, const void *, const void *, int, int, void *, void *, void *);
using AttentionFn = int (*)(const void *, int, int, long long, int, const void *, int, int, int, const void *, const void *, float, int, const void *, int, int, int, int, const void *,
                            int, const void *, const void *, int, int, int, void *, void *, size_t, void *);

bool whole_number(PyObject *o, int *v)
{
    if (!PyLong_Check(o)) return false;                 // (True and False are numbers too)
    const long x = PyLong_AsLong(o);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    *v = (int)x;
    return x == *v;
}
// a [T, heads, d] tensor of bf16 or f32 whose heads follow one another
struct Heads {
    const at::Tensor *t;
    int T, heads, d, f32;
    long long stride;
};
bool heads_of(PyObject *o, Heads *h)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.has_storage() || !t.is_cuda() || t.is_conj() || t.is_neg() || t.dim() != 3) return false;
    const at::ScalarType type = t.scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX || t.size(2) > INT32_MAX || t.numel() == 0) return false;
    *h = {&t, (int)t.size(0), (int)t.size(1), (int)t.size(2), type == at::kFloat, t.size(0) > 1 ? (long long)t.stride(0) : (long long)(t.size(1) * t.size(2))};
    return t.stride(2) == 1 && (t.size(1) == 1 || t.stride(1) == t.size(2));
}
// address of a contiguous tensor of `count` elements of a type
bool whole(PyObject *o, at::ScalarType type, long long count, const void **p)
{
    const at::Tensor *t = ordinary(o);
    if (t == nullptr || t->scalar_type() != type || t->numel() != count) return false;
    *p = t->const_data_ptr();
    return true;
}
bool whole_or_none(PyObject *o, at::ScalarType type, long long count, const void **p)
{
    *p = nullptr;
    return o == Py_None || whole(o, type, count, p);
}
struct Turn {
    const void *table, *positions;
    int rows, dim, pair;
};
bool turn_of(PyObject *rope, PyObject *positions, PyObject *pair, int T, Turn *r)
{
    *r = {};
    if (rope == Py_None) return true;
    const at::Tensor *t = ordinary(rope);
    if (t == nullptr || t->dim() != 2 || t->scalar_type() != at::kFloat || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX || !whole(positions, at::kInt, T, &r->positions)) return false;
    r->table = t->const_data_ptr();
    r->rows = (int)t->size(0);
    r->dim = (int)t->size(1);
    return whole_number(pair, &r->pair);
}
// a pool of pages: address and number of them.  Sizes that the entry points refuse are left to the functions of binding.py
bool pool_of(PyObject *cache, int page_tokens, int heads, int d, const at::Tensor **pool, int *pages)
{
    *pool = ordinary(cache);
    const long long size = (long long)heads * page_tokens * (d + 4);
    if (*pool == nullptr || (*pool)->element_size() != 1 || page_tokens < 16 || page_tokens > 1024 || (page_tokens & (page_tokens - 1)) != 0 || heads < 1 || heads > 65535 || (d != 64 && d != 128) ||
        (*pool)->numel() % size != 0 || (*pool)->numel() / size > INT32_MAX)
        return false;
    *pages = (int)((*pool)->numel() / size);
    return true;
}
void *current_stream() { return reinterpret_cast<void *>(c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream()); }

template <class Call>
PyObject *guarded(Call &&call)
{
    try {
        return call();
    } catch (python_error &e) {
        e.restore();
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *kv4_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Heads k, v;
        Turn r;
        const at::Tensor *pool;
        const void *signs, *slots;
        int page_tokens, pages;
        if (n != 9 || kv4_entry[kAppend] == nullptr || !heads_of(args[0], &k) || !heads_of(args[1], &v) || k.T != v.T || k.heads != v.heads || k.d != v.d || k.f32 != v.f32 ||
            !whole_or_none(args[2], at::kChar, k.d, &signs) || !whole(args[3], at::kInt, k.T, &slots) || !whole_number(args[5], &page_tokens) ||
            !pool_of(args[4], page_tokens, k.heads, k.d, &pool, &pages) || !turn_of(args[6], args[7], args[8], k.T, &r))
            Py_RETURN_NOTIMPLEMENTED;
        const void *kp = k.t->const_data_ptr(), *vp = v.t->const_data_ptr();
        void *cache = pool->data_ptr(), *stream = current_stream();
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = reinterpret_cast<AppendFn>(kv4_entry[kAppend])(kp, vp, k.f32, k.T, k.stride, v.stride, k.heads, k.d, r.table, r.rows, r.dim, r.pair, r.positions, signs, slots, cache,
                                                               pages, page_tokens, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    });
}

PyObject *kv4_read(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Heads k, v;
        const at::Tensor *pool;
        const void *signs, *slots;
        int page_tokens, pages;
        if (n != 6 || kv4_entry[kRead] == nullptr || !heads_of(args[4], &k) || !heads_of(args[5], &v) || k.T != v.T || k.heads != v.heads || k.d != v.d || k.f32 != v.f32 ||
            !k.t->is_contiguous() || !v.t->is_contiguous() || !whole_or_none(args[2], at::kChar, k.d, &signs) || !whole(args[3], at::kInt, k.T, &slots) ||
            !whole_number(args[1], &page_tokens) || !pool_of(args[0], page_tokens, k.heads, k.d, &pool, &pages))
            Py_RETURN_NOTIMPLEMENTED;
        void *kp = k.t->data_ptr(), *vp = v.t->data_ptr(), *stream = current_stream();
        const void *cache = pool->const_data_ptr();
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = reinterpret_cast<ReadFn>(kv4_entry[kRead])(cache, pages, page_tokens, k.heads, k.d, signs, slots, k.T, k.f32, kp, vp, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    });
}

PyObject *kv4_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Heads q, out;
        Turn r;
        const at::Tensor *pool, *table = n == 17 ? ordinary(args[7]) : nullptr, *ws = nullptr;
        const void *signs, *starts, *lens;
        int causal, page_tokens, kv_heads, pages, max_q, max_kv;
        if (table == nullptr || kv4_entry[kAttention] == nullptr || table->dim() != 2 || table->scalar_type() != at::kInt || table->size(0) >= INT32_MAX || table->size(1) > INT32_MAX ||
            !heads_of(args[0], &q) || !heads_of(args[12], &out) || out.f32 || !out.t->is_contiguous() || out.T != q.T || out.heads != q.heads || out.d != q.d ||
            !whole_or_none(args[1], at::kChar, q.d, &signs) || !PyFloat_Check(args[2]) || !whole_number(args[3], &causal) || !whole_number(args[5], &page_tokens) ||
            !whole_number(args[6], &kv_heads) || !pool_of(args[4], page_tokens, kv_heads, q.d, &pool, &pages) || !whole(args[8], at::kInt, table->size(0) + 1, &starts) ||
            !whole(args[9], at::kInt, table->size(0), &lens) || !whole_number(args[10], &max_q) || !whole_number(args[11], &max_kv) || !turn_of(args[14], args[15], args[16], q.T, &r))
            Py_RETURN_NOTIMPLEMENTED;
        if (args[13] != Py_None && (ws = ordinary(args[13])) == nullptr) Py_RETURN_NOTIMPLEMENTED;
        const void *qp = q.t->const_data_ptr(), *cache = pool->const_data_ptr(), *tp = table->const_data_ptr();
        void *op = out.t->data_ptr(), *wp = ws != nullptr ? ws->data_ptr() : nullptr, *stream = current_stream();
        const size_t bytes = ws != nullptr ? (size_t)ws->numel() * ws->element_size() : 0;
        const float scale = (float)PyFloat_AS_DOUBLE(args[2]);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = reinterpret_cast<AttentionFn>(kv4_entry[kAttention])(qp, q.f32, q.T, q.stride, q.heads, r.table, r.rows, r.dim, r.pair, r.positions, signs, scale, causal, cache, pages,
                                                                     page_tokens, kv_heads, q.d, tp, (int)table->size(1), starts, lens, (int)table->size(0), max_q, max_kv, op, wp, bytes,
                                                                     stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    });
}

PyObject *bind_kv4(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "bind_kv4 takes 2 arguments");
        return nullptr;
    }
    const long which = PyLong_AsLong(args[0]);
    void *const address = PyLong_AsVoidPtr(args[1]);
    if (PyErr_Occurred()) return nullptr;
    if (which < 0 || which >= kKv4) {
        PyErr_SetString(PyExc_ValueError, "no such entry point");
        return nullptr;
    }
    kv4_entry[which] = address;
    Py_RETURN_NONE;
}

PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "bind takes 2 arguments");
        return nullptr;
    }
    const long kind = PyLong_AsLong(args[0]);
    void *const address = PyLong_AsVoidPtr(args[1]);
    if (PyErr_Occurred()) return nullptr;
    if (kind < 0 || kind >= kKinds) {
        PyErr_SetString(PyExc_ValueError, "no such kind");
        return nullptr;
    }
    entry[kind] = address;
    Py_RETURN_NONE;
}

using Fast = PyObject *(*)(PyObject *, PyObject *const *, Py_ssize_t);
PyMethodDef method(const char *name, Fast f) { return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}; }
PyMethodDef methods[] = {method("linear", linear), method("bind", bind), method("kv4_append", kv4_append), method("kv4_read", kv4_read), method("kv4_attention", kv4_attention),
                         method("bind_kv4", bind_kv4),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call()
{
    PyObject *const m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", QVGGT_TORCH_VERSION) != 0) {       // binding.py compares it
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
