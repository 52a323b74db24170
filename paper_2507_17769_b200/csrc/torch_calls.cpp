// Append, gather and run of PagedAttention, and its calls of a speculative step, as a CPython extension that takes torch tensors: the checks, the allocation of the
// results and the call into the library in one step.
//
// Iterations of small batches are bound by the host: 15 us of calls beside kernels of 8 to 12.  Of that the allocation of two results
// from Python took 4 us, and the tensors' addresses and checks 1 a call.  Measured (8 decode rows of 512 tokens): run 7.9 -> 5.5 us,
// append 4.1 -> 3.2, the iteration 14.7 -> 11.7; a gather 8.7 -> 6.6.  Tensors of subclasses do not come here (session.py).
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>

#include <cstdint>
#include <cstring>

#include "../../include/polyserve_attn.h"

namespace {

typedef int (*kv_write_fn)(void*, const void*, const void*, const int32_t*, int32_t, const int32_t*, const int32_t*, int32_t, void*);
typedef int (*kv_gather_fn)(const void*, const int32_t*, int32_t, void*, void*, void*);
typedef int (*attn_run_fn)(void*, const void*, const void*, const int32_t*, void*, float*, void*, size_t, void*);
kv_write_fn f_write;
kv_gather_fn f_gather;
attn_run_fn f_run;
decltype(&ps_kv_write_rope) f_write_rope;
decltype(&ps_attn_tree) f_tree;
decltype(&ps_kv_accept) f_accept;
decltype(&ps_kv_read) f_read;

bool count_is(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    return false;
}
// an address, or None, which the library refuses: a closed session's handles are None
bool as_ptr(PyObject* o, void** p) {
    if (o == Py_None) {
        *p = nullptr;
        return true;
    }
    *p = PyLong_AsVoidPtr(o);
    return !(*p == nullptr && PyErr_Occurred());
}
bool as_i64(PyObject* o, int64_t* v) {  // (what has __index__; a truth value is no size to torch either)
    if (PyBool_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "an integer expected, got bool");
        return false;
    }
    *v = PyLong_AsLongLong(o);
    return !(*v == -1 && PyErr_Occurred());
}
bool as_tensor(PyObject* o, const at::Tensor** t) {
    if (THPVariable_Check(o)) {
        *t = &THPVariable_Unpack(o);
        return true;
    }
    PyErr_SetString(PyExc_TypeError, "a tensor expected");
    return false;
}
bool holds(bool what, const char* message) {
    if (!what) PyErr_SetString(PyExc_AssertionError, message);
    return what;
}

// a contiguous int32 array of one entry per request
struct Lengths {
    Py_buffer b;
    bool held = false;
    bool get(PyObject* o) {
        if (PyObject_GetBuffer(o, &b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) return false;
        held = true;
        if (b.ndim >= 1 && b.itemsize == 4 && b.format && strcmp(b.format, "i") == 0) return true;
        PyErr_SetString(PyExc_TypeError, "lengths must be an int32 array");
        return false;
    }
    ~Lengths() {
        if (held) PyBuffer_Release(&b);
    }
};

// The interpreter lock is given back while the library runs and while results are allocated: an allocation may wait for the device, and
// what that waits for may need the interpreter.
struct Unlocked {
    PyThreadState* s = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(s); }
};

PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[7];
    if (!count_is(n, 7)) return nullptr;
    for (int k = 0; k < 7; ++k)
        if (!as_ptr(a[k], &p[k])) return nullptr;
    f_write = (kv_write_fn)p[0];
    f_gather = (kv_gather_fn)p[1];
    f_run = (attn_run_fn)p[2];
    f_write_rope = (decltype(f_write_rope))p[3];
    f_tree = (decltype(f_tree))p[4];
    f_accept = (decltype(f_accept))p[5];
    f_read = (decltype(f_read))p[6];
    Py_RETURN_NONE;
}

// (kv, k, v, block table, max_pages or None, prior, q_len, stream) -> status
PyObject* py_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *kv, *stream;
    const at::Tensor *k, *v, *bt;
    int64_t max_pages;
    Lengths prior, q_len;
    if (!count_is(n, 8) || !as_ptr(a[0], &kv) || !as_tensor(a[1], &k) || !as_tensor(a[2], &v) || !as_tensor(a[3], &bt) || !as_ptr(a[7], &stream)) return nullptr;
    if (a[4] == Py_None) max_pages = bt->size(-1);
    else if (!as_i64(a[4], &max_pages)) return nullptr;
    if (!holds(k->is_contiguous() && v->is_contiguous() && bt->is_contiguous(), "k_new, v_new and the block table must be contiguous")) return nullptr;
    if (max_pages > INT32_MAX || max_pages < INT32_MIN) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
        return nullptr;
    }
    if (!prior.get(a[5]) || !q_len.get(a[6])) return nullptr;
    if (prior.b.shape[0] > q_len.b.shape[0] || prior.b.shape[0] > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "q_len is shorter than prior");
        return nullptr;
    }
    int st;
    {
        Unlocked u;
        st = f_write(kv, k->data_ptr(), v->data_ptr(), (const int32_t*)bt->data_ptr(), (int32_t)max_pages, (const int32_t*)prior.b.buf, (const int32_t*)q_len.b.buf,
                     (int32_t)prior.b.shape[0], stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

PyObject* three(int st, PyObject* x, PyObject* y) {  // (takes both references)
    THPObjectPtr ox(x), oy(y), os(PyLong_FromLong(st));
    if (!ox || !oy || !os) return nullptr;
    PyObject* t = PyTuple_New(3);
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, os.release());
    PyTuple_SET_ITEM(t, 1, ox.release());
    PyTuple_SET_ITEM(t, 2, oy.release());
    return t;
}
PyObject* again(PyObject* o) {
    Py_INCREF(o);
    return o;
}

// (kv, block table row, length, kv heads, head dim, a tensor of the pool's device, stream) -> (status, K, V)
PyObject* py_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *kv, *stream;
    const at::Tensor *bt, *pool;
    int64_t len, hkv, d;
    if (!count_is(n, 7) || !as_ptr(a[0], &kv) || !as_tensor(a[1], &bt) || !as_i64(a[2], &len) || !as_i64(a[3], &hkv) || !as_i64(a[4], &d) || !as_tensor(a[5], &pool) ||
        !as_ptr(a[6], &stream))
        return nullptr;
    if (len > INT32_MAX || len < INT32_MIN) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
        return nullptr;
    }
    at::Tensor k, v;
    int st;
    {
        Unlocked u;
        const auto opts = pool->options().dtype(at::kBFloat16);
        k = at::empty({len, hkv, d}, opts), v = at::empty({len, hkv, d}, opts);
        st = f_gather(kv, (const int32_t*)bt->data_ptr(), (int32_t)len, k.data_ptr(), v.data_ptr(), stream);
    }
    return three(st, THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
    END_HANDLE_TH_ERRORS
}

// (plan, kv, q, block table, out or None, lse or None, want lse, q tokens, q heads, a tensor of the pool's device, workspace, its
// bytes, stream) -> (status, out, lse or None)
PyObject* py_run(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *plan, *kv, *ws, *stream;
    const at::Tensor *q, *bt, *pool;
    int64_t total_q, hq, bytes;
    if (!count_is(n, 13) || !as_ptr(a[0], &plan) || !as_ptr(a[1], &kv) || !as_tensor(a[2], &q) || !as_tensor(a[3], &bt) || !as_i64(a[7], &total_q) ||
        !as_i64(a[8], &hq) || !as_tensor(a[9], &pool) || !as_ptr(a[10], &ws) || !as_i64(a[11], &bytes) || !as_ptr(a[12], &stream))
        return nullptr;
    if (!holds(q->is_contiguous() && q->size(0) == total_q && bt->is_contiguous(), "q must be contiguous with a row per planned token, and the block table contiguous"))
        return nullptr;
    const at::Tensor *given_out = nullptr, *given_lse = nullptr;
    if ((a[4] != Py_None && !as_tensor(a[4], &given_out)) || (a[5] != Py_None && !as_tensor(a[5], &given_lse))) return nullptr;
    at::Tensor out, lse;
    int st;
    {
        Unlocked u;
        if (!given_out) out = at::empty(q->sizes(), q->options());
        if (!given_lse && a[6] == Py_True) lse = at::empty({total_q, hq}, pool->options().dtype(at::kFloat));
        void* const lse_ptr = given_lse ? given_lse->data_ptr() : lse.defined() ? lse.data_ptr() : nullptr;
        st = f_run(plan, kv, q->data_ptr(), (const int32_t*)bt->data_ptr(), given_out ? given_out->data_ptr() : out.data_ptr(), (float*)lse_ptr, ws, (size_t)bytes,
                   stream);
    }
    return three(st, out.defined() ? THPVariable_Wrap(std::move(out)) : again(a[4]), lse.defined() ? THPVariable_Wrap(std::move(lse)) : again(a[5]));
    END_HANDLE_TH_ERRORS
}

// ---- a speculative step: what the library cannot see of its tensors (types, extents, device) is checked here ----

// the two length arrays of a batch, and how many tokens it has
struct Batch {
    Lengths first, len;
    int32_t n = 0;
    int64_t total = 0;
    bool get(PyObject* a, PyObject* b) {
        if (!first.get(a) || !len.get(b)) return false;
        if (first.b.ndim != 1 || len.b.ndim != 1 || first.b.shape[0] != len.b.shape[0] || first.b.shape[0] > INT32_MAX) {
            PyErr_SetString(PyExc_ValueError, "one length a request in both arrays");
            return false;
        }
        n = (int32_t)first.b.shape[0];
        for (int32_t r = 0; r < n; ++r) total += ((const int32_t*)len.b.buf)[r];  // (negative ones are the library's to refuse)
        return true;
    }
    const int32_t* a() const { return (const int32_t*)first.b.buf; }
    const int32_t* b() const { return (const int32_t*)len.b.buf; }
};
bool optional_tensor(PyObject* o, const at::Tensor** t) {
    *t = nullptr;
    return o == Py_None || as_tensor(o, t);
}
// contiguous, of this type and these extents (-1: any), on the pool's device
bool is_array(const at::Tensor* t, at::ScalarType type, std::initializer_list<int64_t> size, const at::Tensor* pool, const char* message) {
    bool good = t->scalar_type() == type && t->dim() == (int64_t)size.size() && t->is_contiguous() && t->device() == pool->device();
    int64_t i = 0;
    for (int64_t s : size) {
        good = good && (s < 0 || t->size(i) == s);
        ++i;
    }
    return holds(good, message);
}
bool is_table(const at::Tensor* t, const Batch& batch, const at::Tensor* pool) {
    return is_array(t, at::kInt, {-1, -1}, pool, "the block table must be a contiguous int32 matrix on the pool's device") &&
           holds(t->size(0) >= batch.n && t->size(1) <= INT32_MAX, "the block table must have a row per request");
}
// [tokens, heads, d] bf16 with packed heads; *stride: elements from a token to the next
bool is_rows(const at::Tensor* t, int64_t tokens, int64_t heads, int64_t d, const at::Tensor* pool, int64_t* stride, const char* message) {
    const bool good = t->scalar_type() == at::kBFloat16 && t->dim() == 3 && t->size(0) == tokens && t->size(1) == heads && t->size(2) == d && t->stride(2) == 1 &&
                      (heads == 1 || t->stride(1) == d) && (tokens <= 1 || t->stride(0) >= heads * d) && t->device() == pool->device();
    *stride = tokens <= 1 ? heads * d : t->stride(0);
    return holds(good, message);
}

// (kv, q, k, v, block table, prior, q_len, cos_sin or None, positions or None, q weight or None, k weight or None, eps, interleaved,
// q_out or None, q heads, kv heads, head dim, pool, stream) -> (status, q_out)
PyObject* py_write_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *kv, *stream;
    const at::Tensor *q, *k, *v, *bt, *cs, *pos, *qw, *kw, *given, *pool;
    int64_t hq, hkv, d;
    Batch batch;
    if (!count_is(n, 19) || !as_ptr(a[0], &kv) || !as_tensor(a[1], &q) || !as_tensor(a[2], &k) || !as_tensor(a[3], &v) || !as_tensor(a[4], &bt) ||
        !batch.get(a[5], a[6]) || !optional_tensor(a[7], &cs) || !optional_tensor(a[8], &pos) || !optional_tensor(a[9], &qw) || !optional_tensor(a[10], &kw) ||
        !optional_tensor(a[13], &given) || !as_i64(a[14], &hq) || !as_i64(a[15], &hkv) || !as_i64(a[16], &d) || !as_tensor(a[17], &pool) || !as_ptr(a[18], &stream))
        return nullptr;
    const double eps = PyFloat_AsDouble(a[11]);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    const int interleaved = PyObject_IsTrue(a[12]);
    if (interleaved < 0) return nullptr;
    ps_rope r{};
    const int64_t T = batch.total;
    if (!is_rows(q, T, hq, d, pool, &r.q_stride, "q must be bf16 [tokens, q heads, head dim] with packed heads, on the pool's device") ||
        !is_rows(k, T, hkv, d, pool, &r.k_stride, "k_new must be bf16 [tokens, kv heads, head dim] with packed heads, on the pool's device") ||
        !is_rows(v, T, hkv, d, pool, &r.v_stride, "v_new must be bf16 [tokens, kv heads, head dim] with packed heads, on the pool's device") || !is_table(bt, batch, pool) ||
        (cs && !is_array(cs, at::kFloat, {-1, -1}, pool, "cos_sin must be a contiguous float32 matrix on the pool's device")) ||
        (pos && !is_array(pos, at::kInt, {T}, pool, "positions must be contiguous int32 [tokens] on the pool's device")) ||
        (qw && !is_array(qw, at::kBFloat16, {d}, pool, "q_weight must be contiguous bf16 [head dim] on the pool's device")) ||
        (kw && !is_array(kw, at::kBFloat16, {d}, pool, "k_weight must be contiguous bf16 [head dim] on the pool's device")) ||
        (given && !is_array(given, at::kBFloat16, {T, hq, d}, pool, "q_out must be contiguous bf16 [tokens, q heads, head dim] on the pool's device")) ||
        (cs && !holds(cs->size(1) <= INT32_MAX, "cos_sin is too wide")))
        return nullptr;
    at::Tensor out;
    int st;
    {
        Unlocked u;
        const c10::DeviceGuard there(pool->device());  // (a stream takes launches while its device is the current one)
        if (!given) out = at::empty({T, hq, d}, pool->options().dtype(at::kBFloat16));
        r.q_dev = q->data_ptr(), r.k_new_dev = k->data_ptr(), r.v_new_dev = v->data_ptr();
        r.q_out_dev = given ? given->data_ptr() : out.data_ptr();
        r.q_weight_dev = qw ? qw->data_ptr() : nullptr;
        r.k_weight_dev = kw ? kw->data_ptr() : nullptr;
        r.cos_sin_dev = cs ? (const float*)cs->data_ptr() : nullptr;
        r.n_positions = cs ? cs->size(0) : 0;
        r.rot_dim = cs ? (int32_t)cs->size(1) : 0;
        r.positions_dev = pos ? (const int32_t*)pos->data_ptr() : nullptr;
        r.interleaved = interleaved;
        r.eps = (float)eps;
        st = f_write_rope((ps_kv*)kv, &r, (const int32_t*)bt->data_ptr(), (int32_t)bt->size(1), batch.a(), batch.b(), batch.n, stream);
    }
    PyObject* const got = given ? again(a[13]) : THPVariable_Wrap(std::move(out));
    return got ? Py_BuildValue("iN", st, got) : nullptr;
    END_HANDLE_TH_ERRORS
}

// (kv, q, block table, mask, prior, n_nodes, out or None, lse or None, want lse, q heads, head dim, pool, bytes of workspace, stream)
// -> (status, out, lse or None).  The workspace is the call's own, from the stream's memory, as its results are: calls on several streams, and
// graphs that are replayed side by side, share none.
PyObject* py_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *kv, *stream;
    const at::Tensor *q, *bt, *mask, *given_out, *given_lse, *pool;
    int64_t hq, d, bytes;
    Batch batch;
    if (!count_is(n, 14) || !as_ptr(a[0], &kv) || !as_tensor(a[1], &q) || !as_tensor(a[2], &bt) || !as_tensor(a[3], &mask) || !batch.get(a[4], a[5]) ||
        !optional_tensor(a[6], &given_out) || !optional_tensor(a[7], &given_lse) || !as_i64(a[9], &hq) || !as_i64(a[10], &d) || !as_tensor(a[11], &pool) ||
        !as_i64(a[12], &bytes) || !as_ptr(a[13], &stream))
        return nullptr;
    const int64_t T = batch.total;
    if (!is_array(q, at::kBFloat16, {T, hq, d}, pool, "q must be contiguous bf16 [tokens, q heads, head dim] on the pool's device") || !is_table(bt, batch, pool) ||
        !is_array(mask, at::kLong, {T, -1}, pool, "mask must be contiguous int64 [tokens, words] on the pool's device") ||
        !holds(mask->size(1) <= INT32_MAX, "mask is too wide") ||
        (given_out && !is_array(given_out, at::kBFloat16, {T, hq, d}, pool, "out must be contiguous bf16 [tokens, q heads, head dim] on the pool's device")) ||
        (given_lse && !is_array(given_lse, at::kFloat, {T, hq}, pool, "lse must be contiguous float32 [tokens, q heads] on the pool's device")))
        return nullptr;
    at::Tensor out, lse;
    int st;
    {
        Unlocked u;
        const c10::DeviceGuard there(pool->device());  // (a stream takes launches while its device is the current one)
        if (!given_out) out = at::empty({T, hq, d}, q->options());
        if (!given_lse && a[8] == Py_True) lse = at::empty({T, hq}, pool->options().dtype(at::kFloat));
        void* const lse_ptr = given_lse ? given_lse->data_ptr() : lse.defined() ? lse.data_ptr() : nullptr;
        const at::Tensor ws = at::empty({bytes + 256}, pool->options().dtype(at::kByte));
        void* const ws_ptr = (void*)(((uintptr_t)ws.data_ptr() + 255) / 256 * 256);
        st = f_tree((const ps_kv*)kv, q->data_ptr(), (const int32_t*)bt->data_ptr(), (int32_t)bt->size(1), (const int64_t*)mask->data_ptr(), (int32_t)mask->size(1),
                    batch.a(), batch.b(), batch.n, given_out ? given_out->data_ptr() : out.data_ptr(), (float*)lse_ptr, ws_ptr, (size_t)bytes, stream);
    }
    return three(st, out.defined() ? THPVariable_Wrap(std::move(out)) : again(a[6]), lse.defined() ? THPVariable_Wrap(std::move(lse)) : again(a[7]));
    END_HANDLE_TH_ERRORS
}

// (kv, block table, prior, n_nodes, index, count, pool, stream) -> status
PyObject* py_accept(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *kv, *stream;
    const at::Tensor *bt, *index, *count, *pool;
    Batch batch;
    if (!count_is(n, 8) || !as_ptr(a[0], &kv) || !as_tensor(a[1], &bt) || !batch.get(a[2], a[3]) || !as_tensor(a[4], &index) || !as_tensor(a[5], &count) ||
        !as_tensor(a[6], &pool) || !as_ptr(a[7], &stream))
        return nullptr;
    if (!is_table(bt, batch, pool) || !is_array(index, at::kInt, {batch.n, -1}, pool, "index must be contiguous int32 [requests, width] on the pool's device") ||
        !holds(index->size(1) <= INT32_MAX, "index is too wide") || !is_array(count, at::kInt, {batch.n}, pool, "count must be contiguous int32 [requests] on the pool's device"))
        return nullptr;
    int st;
    {
        Unlocked u;
        const c10::DeviceGuard there(pool->device());  // (a stream takes launches while its device is the current one)
        st = f_accept((ps_kv*)kv, (const int32_t*)bt->data_ptr(), (int32_t)bt->size(1), batch.a(), batch.b(), batch.n, (const int32_t*)index->data_ptr(),
                      (int32_t)index->size(1), (const int32_t*)count->data_ptr(), stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// (kv, block table, begin, length, kv heads, head dim, pool, stream) -> (status, K, V)
PyObject* py_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    void *kv, *stream;
    const at::Tensor *bt, *pool;
    int64_t hkv, d;
    Batch batch;
    if (!count_is(n, 8) || !as_ptr(a[0], &kv) || !as_tensor(a[1], &bt) || !batch.get(a[2], a[3]) || !as_i64(a[4], &hkv) || !as_i64(a[5], &d) || !as_tensor(a[6], &pool) ||
        !as_ptr(a[7], &stream))
        return nullptr;
    if (!is_table(bt, batch, pool)) return nullptr;
    at::Tensor k, v;
    int st;
    {
        Unlocked u;
        const c10::DeviceGuard there(pool->device());  // (a stream takes launches while its device is the current one)
        const auto read = [&](void* k_out, void* v_out) {
            return f_read((const ps_kv*)kv, (const int32_t*)bt->data_ptr(), (int32_t)bt->size(1), batch.a(), batch.b(), batch.n, k_out, v_out, stream);
        };
        st = read(nullptr, nullptr);  // (the library's checks: lengths that it refuses may ask for any amount of memory)
        if (st == PS_OK) {
            const auto opts = pool->options().dtype(at::kBFloat16);
            k = at::empty({batch.total, hkv, d}, opts), v = at::empty({batch.total, hkv, d}, opts);
            st = read(k.data_ptr(), v.data_ptr());
        }
    }
    if (!k.defined()) return three(st, again(Py_None), again(Py_None));
    return three(st, THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, "addresses of the library's functions"},
    {"write_rope", (PyCFunction)(void (*)(void))py_write_rope, METH_FASTCALL, "ps_kv_write_rope"},
    {"tree", (PyCFunction)(void (*)(void))py_tree, METH_FASTCALL, "ps_attn_tree"},
    {"accept", (PyCFunction)(void (*)(void))py_accept, METH_FASTCALL, "ps_kv_accept"},
    {"read", (PyCFunction)(void (*)(void))py_read, METH_FASTCALL, "ps_kv_read into new tensors"},
    {"write", (PyCFunction)(void (*)(void))py_write, METH_FASTCALL, "ps_kv_write"},
    {"gather", (PyCFunction)(void (*)(void))py_gather, METH_FASTCALL, "ps_kv_gather into new tensors"},
    {"run", (PyCFunction)(void (*)(void))py_run, METH_FASTCALL, "ps_attn_run"},
    {nullptr, nullptr, 0, nullptr},
};
struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&module); }
