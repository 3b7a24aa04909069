// CPython module _lychee_torch: argument marshalling of the per-token entry points for torch tensors.
//
// A decode step at a short context is shorter on the GPU than its call was in Python: ctypes
// conversions, tensor accessors and the current-stream object took about half of the 12.9 us a call spent on the
// host.  Here the tensors are read through torch's C++ objects.  The module calls the C ABI through the
// addresses the binding hands over (bind), so it works with whichever build of the library is loaded.
// A call with arguments that are no tensors returns NotImplemented and the binding marshals it itself.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>

#include <climits>
#include <exception>
#include <initializer_list>

#include "lychee.h"

namespace {

decltype(&lc_decode_step) g_decode_step = nullptr;
decltype(&lc_decode_step_static) g_decode_step_static = nullptr;
decltype(&lc_retrieve) g_retrieve = nullptr;
decltype(&lc_sparse_decode) g_sparse_decode = nullptr;
decltype(&lc_append) g_append = nullptr;
decltype(&lc_cache4_store) g_cache4_store = nullptr;
decltype(&lc_cache4_load) g_cache4_load = nullptr;
decltype(&lc_sparse_decode4) g_sparse_decode4 = nullptr;
decltype(&lc_append4) g_append4 = nullptr;
decltype(&lc_weigh_chunks) g_weigh_chunks = nullptr;
decltype(&lc_weigh_chunks4) g_weigh_chunks4 = nullptr;
decltype(&lc_evict_select) g_evict_select = nullptr;
decltype(&lc_evict_rows) g_evict_rows = nullptr;
decltype(&lc_evict_rows4) g_evict_rows4 = nullptr;

// The entry points of the 4-bit cache and of the eviction.
PyObject* bind4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "bind4(cache4_store, cache4_load, sparse_decode4, append4, weigh_chunks, weigh_chunks4, evict_select, evict_rows, evict_rows4)");
        return nullptr;
    }
    g_cache4_store = reinterpret_cast<decltype(g_cache4_store)>(PyLong_AsVoidPtr(a[0]));
    g_cache4_load = reinterpret_cast<decltype(g_cache4_load)>(PyLong_AsVoidPtr(a[1]));
    g_sparse_decode4 = reinterpret_cast<decltype(g_sparse_decode4)>(PyLong_AsVoidPtr(a[2]));
    g_append4 = reinterpret_cast<decltype(g_append4)>(PyLong_AsVoidPtr(a[3]));
    g_weigh_chunks = reinterpret_cast<decltype(g_weigh_chunks)>(PyLong_AsVoidPtr(a[4]));
    g_weigh_chunks4 = reinterpret_cast<decltype(g_weigh_chunks4)>(PyLong_AsVoidPtr(a[5]));
    g_evict_select = reinterpret_cast<decltype(g_evict_select)>(PyLong_AsVoidPtr(a[6]));
    g_evict_rows = reinterpret_cast<decltype(g_evict_rows)>(PyLong_AsVoidPtr(a[7]));
    g_evict_rows4 = reinterpret_cast<decltype(g_evict_rows4)>(PyLong_AsVoidPtr(a[8]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind(decode_step, decode_step_static, retrieve, sparse_decode, append)");
        return nullptr;
    }
    g_decode_step = reinterpret_cast<decltype(g_decode_step)>(PyLong_AsVoidPtr(a[0]));
    g_decode_step_static = reinterpret_cast<decltype(g_decode_step_static)>(PyLong_AsVoidPtr(a[1]));
    g_retrieve = reinterpret_cast<decltype(g_retrieve)>(PyLong_AsVoidPtr(a[2]));
    g_sparse_decode = reinterpret_cast<decltype(g_sparse_decode)>(PyLong_AsVoidPtr(a[3]));
    g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[4]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// What the index has room for: {sequences, KV heads, chunks, tokens}; not known of an object that carries a handle alone.
struct Room {
    bool known = false;
    int64_t n[4] = {0, 0, 0, 0};
    int64_t B() const { return n[0]; }
    int64_t H() const { return n[1]; }
    int64_t chunks() const { return n[2]; }
    int64_t tokens() const { return n[3]; }
};

// Positional arguments of one call.
class Args {
  public:
    Args(PyObject* const* a, Py_ssize_t n) : a_(a), n_(n) {}
    bool count(Py_ssize_t n) {
        if (n_ == n) return true;
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", n, n_);
        return false;
    }
    // The tensor at i, or null for None; anything else makes the call not ours.
    const at::Tensor* tensor(int i) {
        if (a_[i] == Py_None) return nullptr;
        if (!THPVariable_Check(a_[i])) { foreign_ = true; return nullptr; }
        return &THPVariable_Unpack(a_[i]);
    }
    void* ptr(int i) {
        const at::Tensor* t = tensor(i);
        return t ? t->data_ptr() : nullptr;
    }
    // What int(x) gives, in C's int (as ctypes passes it: the low 32 bits).
    int integer(int i) {
        PyObject* const v = PyLong_CheckExact(a_[i]) ? Py_NewRef(a_[i]) : PyNumber_Long(a_[i]);
        const int r = v ? (int)PyLong_AsUnsignedLongMask(v) : -1;
        Py_XDECREF(v);
        return r;
    }
    // What int(x) gives, in C's int or the end of its range that is nearest.
    int limited(int i) {
        PyObject* const v = PyNumber_Long(a_[i]);
        int over = 0;
        const long r = v ? PyLong_AsLongAndOverflow(v, &over) : -1;
        Py_XDECREF(v);
        if (over > 0 || r > INT_MAX) return INT_MAX;
        return over < 0 || r < INT_MIN ? INT_MIN : (int)r;
    }
    // integer() of an integer alone; a float or a text makes the call not ours (ctypes refuses it).
    int whole(int i) {
        if (!PyIndex_Check(a_[i])) { foreign_ = true; return -1; }
        PyObject* const v = PyNumber_Index(a_[i]);
        const int r = v ? (int)PyLong_AsUnsignedLongMask(v) : -1;
        Py_XDECREF(v);
        return r;
    }
    Room room(int i) {
        Room r;
        if (!PyTuple_Check(a_[i]) || PyTuple_GET_SIZE(a_[i]) != 4) return r;
        for (int k = 0; k < 4; ++k) r.n[k] = PyLong_AsLong(PyTuple_GET_ITEM(a_[i], k));
        r.known = !PyErr_Occurred();
        return r;
    }
    lc_index* handle(int i) { return static_cast<lc_index*>(PyLong_AsVoidPtr(a_[i])); }
    void* stream(int i) {
        if (a_[i] == Py_None) return c10::hip::getCurrentHIPStream().stream();
        PyObject* const v = PyObject_GetAttrString(a_[i], "cuda_stream");
        void* const s = v ? PyLong_AsVoidPtr(v) : nullptr;
        Py_XDECREF(v);
        return s;
    }
    PyObject* operator[](int i) const { return a_[i]; }
    bool foreign() const { return foreign_; }

  private:
    PyObject* const* a_;
    Py_ssize_t n_;
    bool foreign_ = false;
};

bool cache_strides(const at::Tensor& K, const at::Tensor& V, bool shapes, int64_t (&s)[3]) {
    if ((shapes && !K.sizes().equals(V.sizes())) || !K.strides().equals(V.strides())) {
        PyErr_SetString(PyExc_AssertionError, "K and V must have the same shape and strides");
        return false;
    }
    if (K.dim() != 4 || K.stride(3) != 1) {
        PyErr_SetString(PyExc_AssertionError, "cache must be [B][H_kv][tokens][d] with d contiguous");
        return false;
    }
    for (int i = 0; i < 3; ++i) s[i] = K.stride(i);
    return true;
}
// The interpreter is free for other threads while a call is in the library, as it is under ctypes: a launch can block
// (a full hardware queue).  Everything the call needs has been read from the Python objects before.
class Unlocked {
  public:
    Unlocked() : state_(PyEval_SaveThread()) {}
    ~Unlocked() { PyEval_RestoreThread(state_); }
    Unlocked(const Unlocked&) = delete;
    Unlocked& operator=(const Unlocked&) = delete;

  private:
    PyThreadState* state_;
};
size_t bytes(const at::Tensor& t) { return (size_t)t.numel() * t.element_size(); }

// The result of a call, or NotImplemented / the pending Python error.
template <typename F>
PyObject* guarded(Args& a, F call) {
    try {
        int rc = 0;
        const bool done = call(&rc);
        if (PyErr_Occurred()) return nullptr;
        if (a.foreign() || !done) Py_RETURN_NOTIMPLEMENTED;
        return PyLong_FromLong(rc);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// decode_step(handle, q, K, V, budget, out, ws or None, lse, chunk_ids, counts, stream, static)
PyObject* decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(12)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *q = a.tensor(1), *K = a.tensor(2), *V = a.tensor(3), *ws = a.tensor(6), *ids = a.tensor(8);
        const bool fixed = a[11] == Py_True;
        if (!q || !K || !V || (!fixed && !ws) || a.foreign()) return false;
        int64_t s[3];
        if (!cache_strides(*K, *V, true, s)) return true;
        const int budget = a.integer(4), cap = ids ? (int)ids->size(-1) : 0;
        float* const out = static_cast<float*>(a.ptr(5));
        float* const lse = static_cast<float*>(a.ptr(7));
        int32_t* const counts = static_cast<int32_t*>(a.ptr(9));
        if (PyErr_Occurred() || a.foreign()) return false;
        int32_t* const idp = ids ? static_cast<int32_t*>(ids->data_ptr()) : nullptr;
        void* const st = a.stream(10);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const void *qd = q->data_ptr(), *kd = K->data_ptr(), *vd = V->data_ptr();
        void* const wd = fixed ? nullptr : ws->data_ptr();
        const size_t wn = fixed ? 0 : bytes(*ws);
        const int H_q = (int)q->size(1);
        const Unlocked unlocked;
        *rc = fixed ? g_decode_step_static(idx, qd, kd, vd, s, H_q, budget, out, lse, idp, counts, cap, st)
                    : g_decode_step(idx, qd, kd, vd, s, H_q, budget, out, lse, idp, counts, cap, wd, wn, st);
        return true;
    });
}

// retrieve(handle, q, budget, chunk_ids, counts, ws, scores, stream)
PyObject* retrieve(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(8)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *q = a.tensor(1), *ids = a.tensor(3), *ws = a.tensor(5);
        if (!q || !ids || !ws || a.foreign()) return false;
        const int budget = a.whole(2);
        int32_t* const counts = static_cast<int32_t*>(a.ptr(4));
        float* const scores = static_cast<float*>(a.ptr(6));
        if (PyErr_Occurred() || a.foreign()) return false;
        void* const st = a.stream(7);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const void* const qd = q->data_ptr();
        int32_t* const idp = static_cast<int32_t*>(ids->data_ptr());
        const int H_q = (int)q->size(1), cap = (int)ids->size(2);
        void* const wd = ws->data_ptr();
        const size_t wn = bytes(*ws);
        const Unlocked unlocked;
        *rc = g_retrieve(idx, qd, H_q, budget, idp, counts, scores, cap, wd, wn, st);
        return true;
    });
}

// sparse_decode(handle, q, K, V, chunk_ids, counts, out, ws, lse, stream)
PyObject* sparse_decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(10)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *q = a.tensor(1), *K = a.tensor(2), *V = a.tensor(3), *ids = a.tensor(4), *ws = a.tensor(7);
        if (!q || !K || !V || !ids || !ws || a.foreign()) return false;
        int64_t s[3];
        if (!cache_strides(*K, *V, false, s)) return true;
        const int32_t* const counts = static_cast<const int32_t*>(a.ptr(5));
        float* const out = static_cast<float*>(a.ptr(6));
        float* const lse = static_cast<float*>(a.ptr(8));
        if (a.foreign()) return false;
        void* const st = a.stream(9);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const void *qd = q->data_ptr(), *kd = K->data_ptr(), *vd = V->data_ptr();
        const int32_t* const idp = static_cast<const int32_t*>(ids->data_ptr());
        const int H_q = (int)q->size(1), cap = (int)ids->size(2);
        void* const wd = ws->data_ptr();
        const size_t wn = bytes(*ws);
        const Unlocked unlocked;
        *rc = g_sparse_decode(idx, qd, kd, vd, s, idp, counts, cap, H_q, out, lse, wd, wn, st);
        return true;
    });
}

// The close flags of an append: truth values of a sized iterable.
bool close_flags(PyObject* given, uint8_t (&flags)[1024]) {
    // (a tuple of its own: telling whether an element is true can run code that changes the caller's list)
    PyObject* const seq = PyObject_Size(given) >= 0 ? PySequence_Tuple(given) : nullptr;
    if (!seq) return false;
    const Py_ssize_t m = PyTuple_GET_SIZE(seq);
    bool ok = m <= (Py_ssize_t)sizeof(flags);
    for (Py_ssize_t i = 0; ok && i < m; ++i) {
        const int t = PyObject_IsTrue(PyTuple_GET_ITEM(seq, i));
        if (t < 0) ok = false;
        else flags[i] = (uint8_t)t;
    }
    Py_DECREF(seq);
    return ok;
}

// append(handle, K, V, k_new, v_new, close flags or None, ws, stream)
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(8)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *K = a.tensor(1), *V = a.tensor(2), *k = a.tensor(3), *v = a.tensor(4), *ws = a.tensor(6);
        if (!K || !V || !k || !v || !ws || a.foreign()) return false;
        int64_t s[3];
        if (!cache_strides(*K, *V, false, s)) return true;
        uint8_t flags[1024] = {};                            // lc_append takes at most 1024 sequences
        const bool given = a[5] != Py_None;
        if (given && !close_flags(a[5], flags)) return false;
        void* const st = a.stream(7);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        void *kd = K->data_ptr(), *vd = V->data_ptr();
        const void *kn = k->data_ptr(), *vn = v->data_ptr();
        void* const wd = ws->data_ptr();
        const size_t wn = bytes(*ws);
        const Unlocked unlocked;
        *rc = g_append(idx, kd, vd, s, kn, vn, given ? flags : nullptr, wd, wn, st);
        return true;
    });
}

// Whether the tensors hold bfloat16 values, or their bits in an integer type.
bool bfloat16s(std::initializer_list<const at::Tensor*> tensors) {
    for (const at::Tensor* t : tensors)
        if (t->element_size() != 2 || t->scalar_type() == at::kHalf) {
            PyErr_SetString(PyExc_AssertionError, "queries, keys and values must be bfloat16");
            return false;
        }
    return true;
}

// Strides of a 4-bit cache, in bytes.
bool cache4_strides(const at::Tensor& K4, const at::Tensor& V4, int64_t (&s)[3]) {
    if (!K4.sizes().equals(V4.sizes()) || !K4.strides().equals(V4.strides())) {
        PyErr_SetString(PyExc_AssertionError, "K4 and V4 must have the same shape and strides");
        return false;
    }
    if (K4.dim() != 4 || K4.size(3) != LC_CACHE4_ROW || K4.stride(3) != 1 || K4.element_size() != 1 || V4.element_size() != 1) {
        PyErr_SetString(PyExc_AssertionError, "4-bit cache must be uint8 [B][H_kv][tokens][68] with a row's bytes contiguous");
        return false;
    }
    for (int i = 0; i < 3; ++i) s[i] = K4.stride(i);
    return true;
}
// At most N whole numbers of a sequence into `to`; false without a Python error: not ours.
template <size_t N>
bool numbers(PyObject* given, Py_ssize_t n, int32_t (&to)[N]) {
    PyObject* const seq = PySequence_Tuple(given);
    if (!seq) { PyErr_Clear(); return false; }
    bool ok = PyTuple_GET_SIZE(seq) == n && n <= (Py_ssize_t)N;
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
        const long v = PyLong_AsLong(PyTuple_GET_ITEM(seq, i));
        ok = !PyErr_Occurred() && v >= -0x7fffffffL && v <= 0x7fffffffL;
        to[i] = (int32_t)v;
    }
    PyErr_Clear();
    Py_DECREF(seq);
    return ok;
}

// move4(store, K, V, K4, V4, first or None, counts or None, stream): lc_cache4_store or lc_cache4_load.  What is unusual (a wrong shape among it)
// is left to the binding's own route.
PyObject* move4(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(8)) return nullptr;
    return guarded(a, [&](int* rc) {
        const bool store = a[0] == Py_True;
        const at::Tensor *K = a.tensor(1), *V = a.tensor(2), *K4 = a.tensor(3), *V4 = a.tensor(4);
        if (!K || !V || !K4 || !V4 || a.foreign()) return false;
        if (K->dim() != 4 || K4->dim() != 4 || K->element_size() != 2 || V->element_size() != 2 || !K->sizes().equals(V->sizes()) || !K4->sizes().equals(V4->sizes()) ||
            K->size(0) != K4->size(0) || K->size(1) != K4->size(1) || K->size(0) > 256 || K->size(2) > 0x7fffffffL || K4->size(2) > 0x7fffffffL)
            return false;
        if (!bfloat16s({K, V})) return true;
        int64_t s[3], s4[3];
        if (!cache_strides(*K, *V, true, s) || !cache4_strides(*K4, *V4, s4)) return true;
        const int B = (int)K->size(0), H = (int)K->size(1), rows = (int)K->size(2), d = (int)K->size(3);
        int32_t first[256], counts[256];
        const bool given = a[5] != Py_None;
        if (given && !numbers(a[5], B, first)) return false;
        if (a[6] == Py_None) {
            for (int b = 0; b < B; ++b) counts[b] = rows;
        } else if (!numbers(a[6], B, counts)) {
            return false;
        }
        for (int b = 0; b < B; ++b)
            if (counts[b] > rows) return false;
        void* const st = a.stream(7);
        if (PyErr_Occurred()) return false;
        void *kd = K->data_ptr(), *vd = V->data_ptr(), *k4 = K4->data_ptr(), *v4 = V4->data_ptr();
        const int cap = (int)K4->size(2);
        const Unlocked unlocked;
        *rc = store ? g_cache4_store(kd, vd, s, given ? first : nullptr, counts, B, H, d, k4, v4, s4, cap, st)
                    : g_cache4_load(k4, v4, s4, given ? first : nullptr, counts, B, H, d, kd, vd, s, cap, st);
        return true;
    });
}

// Whether t, if there is one, holds `rows` rows of `row` 32-bit numbers one behind the other (row 0: that many numbers).  With exactly as many numbers, or a single
// row, the shape says nothing; of a larger table the rows have to be of that length.
bool table(const at::Tensor* t, bool floats, int64_t rows, int64_t row, const char* name) {
    if (!t || (t->is_contiguous() && t->element_size() == 4 && t->is_floating_point() == floats && t->numel() >= rows * (row ? row : 1) &&
               (row == 0 || rows == 1 || t->numel() == rows * row || t->dim() < 2 || t->size(-1) == row)))
        return true;
    PyErr_Format(PyExc_AssertionError, "%s must be a contiguous %s table with the index's room", name, floats ? "float32" : "int32");
    return false;
}

// Whether an input holds n values one behind the other.
bool dense(const at::Tensor& t, int64_t n, const char* name) {
    if (t.is_contiguous() && t.numel() >= n) return true;
    PyErr_Format(PyExc_AssertionError, "%s must be contiguous and hold the index's sequences and heads", name);
    return false;
}
// Whether a cache (of four dimensions) has the index's sequences and heads, and `rows` rows.
bool holds(const at::Tensor& K, const Room& room, int64_t rows) {
    if (K.size(0) >= room.B() && K.size(1) >= room.H() && K.size(2) >= rows) return true;
    PyErr_SetString(PyExc_AssertionError, "the cache must have the index's sequences and heads, and max_tokens rows where it is appended to");
    return false;
}

// sparse_decode4(handle, q, K4, V4, chunk_ids, counts, out, ws, lse, stream, room)
PyObject* sparse_decode4(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(11)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *q = a.tensor(1), *K = a.tensor(2), *V = a.tensor(3), *ids = a.tensor(4), *ws = a.tensor(7);
        if (!q || !K || !V || !ids || !ws || a.foreign()) return false;
        int64_t s[3];
        if (!bfloat16s({q}) || !cache4_strides(*K, *V, s)) return true;
        const at::Tensor *n_t = a.tensor(5), *out_t = a.tensor(6), *lse_t = a.tensor(8);
        const Room room = a.room(10);
        if (room.known) {
            const int64_t pairs = room.B() * room.H(), values = room.B() * q->size(1) * LC_HEAD_DIM;
            if (!dense(*q, values, "q") || !holds(*K, room, 0) || !table(ids, false, pairs, ids->size(-1), "chunk_ids") || !table(n_t, false, pairs, 0, "counts") ||
                !table(out_t, true, values, 0, "out") || !table(lse_t, true, room.B(), q->size(1), "lse"))
                return true;
        }
        const int32_t* const counts = static_cast<const int32_t*>(a.ptr(5));
        float* const out = static_cast<float*>(a.ptr(6));
        float* const lse = static_cast<float*>(a.ptr(8));
        if (a.foreign()) return false;
        void* const st = a.stream(9);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const void *qd = q->data_ptr(), *kd = K->data_ptr(), *vd = V->data_ptr();
        const int32_t* const idp = static_cast<const int32_t*>(ids->data_ptr());
        const int H_q = (int)q->size(1), cap = (int)ids->size(2);
        void* const wd = ws->data_ptr();
        const size_t wn = bytes(*ws);
        const Unlocked unlocked;
        *rc = g_sparse_decode4(idx, qd, kd, vd, s, idp, counts, cap, H_q, out, lse, wd, wn, st);
        return true;
    });
}

// append4(handle, K4, V4, k_new, v_new, close flags or None, stream, room)
PyObject* append4(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(8)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *K = a.tensor(1), *V = a.tensor(2), *k = a.tensor(3), *v = a.tensor(4);
        if (!K || !V || !k || !v || a.foreign()) return false;
        int64_t s[3];
        if (!bfloat16s({k, v}) || !cache4_strides(*K, *V, s)) return true;
        const Room room = a.room(7);
        if (room.known) {
            const int64_t values = room.B() * room.H() * LC_HEAD_DIM;
            if (!holds(*K, room, room.tokens()) || !dense(*k, values, "k_new") || !dense(*v, values, "v_new")) return true;
        }
        uint8_t flags[1024] = {};                            // lc_append4 takes at most 1024 sequences
        const bool given = a[5] != Py_None;
        if (given && !close_flags(a[5], flags)) return false;
        void* const st = a.stream(6);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        void *kd = K->data_ptr(), *vd = V->data_ptr();
        const void *kn = k->data_ptr(), *vn = v->data_ptr();
        const Unlocked unlocked;
        *rc = g_append4(idx, kd, vd, s, kn, vn, given ? flags : nullptr, st);
        return true;
    });
}

// The lists of the chunks that stay.
bool keep_tables(const Room& room, const at::Tensor* ids, const at::Tensor* bounds, const at::Tensor* counts) {
    return !room.known || (table(ids, false, room.B(), room.chunks(), "keep_ids") && table(bounds, false, room.B(), room.chunks() + 1, "keep_bounds") &&
                           table(counts, false, room.B(), 0, "keep_counts"));
}

// weigh_chunks(handle, q, K or K4, chunk_ids, counts, lse, weights, stream, in 4 bits, room)
PyObject* weigh_chunks(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(10)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *q = a.tensor(1), *K = a.tensor(2), *ids = a.tensor(3), *n_t = a.tensor(4), *lse_t = a.tensor(5), *w_t = a.tensor(6);
        const bool in4 = a[8] == Py_True;
        if (!q || !K || !ids || a.foreign()) return false;
        int64_t s[3];
        if (!bfloat16s({q}) || (in4 ? !cache4_strides(*K, *K, s) : !bfloat16s({K}) || !cache_strides(*K, *K, false, s))) return true;
        const Room room = a.room(9);
        if (room.known) {
            const int64_t pairs = room.B() * room.H();
            if (!dense(*q, room.B() * q->size(1) * LC_HEAD_DIM, "q") || !holds(*K, room, 0) ||
                !table(ids, false, pairs, ids->size(-1), "chunk_ids") || !table(n_t, false, pairs, 0, "counts") || !table(lse_t, true, room.B(), q->size(1), "lse") || !table(w_t, true, pairs, room.chunks(), "weights"))
                return true;
        }
        const int32_t* const counts = static_cast<const int32_t*>(a.ptr(4));
        const float* const lse = static_cast<const float*>(a.ptr(5));
        float* const weights = static_cast<float*>(a.ptr(6));
        if (a.foreign()) return false;
        void* const st = a.stream(7);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const void *qd = q->data_ptr(), *kd = K->data_ptr();
        const int32_t* const idp = static_cast<const int32_t*>(ids->data_ptr());
        const int H_q = (int)q->size(1), cap = (int)ids->size(2);
        const Unlocked unlocked;
        *rc = (in4 ? g_weigh_chunks4 : g_weigh_chunks)(idx, qd, kd, s, idp, counts, cap, H_q, lse, weights, st);
        return true;
    });
}

// evict_select(handle, weights, keep_tokens, recent_tokens, keep_ids, keep_bounds, keep_counts, ws, keep_lens, stream, room)
PyObject* evict_select(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(11)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *w = a.tensor(1), *ids_t = a.tensor(4), *bounds_t = a.tensor(5), *n_t = a.tensor(6), *ws = a.tensor(7), *lens_t = a.tensor(8);
        if (!w || !ws || a.foreign()) return false;
        const Room room = a.room(10);
        if (!keep_tables(room, ids_t, bounds_t, n_t)) return true;
        if (room.known && (!table(w, true, room.B() * room.H(), room.chunks(), "weights") || !table(lens_t, false, room.B(), 0, "keep_lens"))) return true;
        const int keep = a.limited(2), recent = a.limited(3);
        if (PyErr_Occurred()) return false;
        int32_t* const ids = static_cast<int32_t*>(a.ptr(4));
        int32_t* const bounds = static_cast<int32_t*>(a.ptr(5));
        int32_t* const counts = static_cast<int32_t*>(a.ptr(6));
        int32_t* const lens = static_cast<int32_t*>(a.ptr(8));
        if (a.foreign()) return false;
        void* const st = a.stream(9);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const float* const wd = static_cast<const float*>(w->data_ptr());
        void* const sd = ws->data_ptr();
        const size_t sn = bytes(*ws);
        const Unlocked unlocked;
        *rc = g_evict_select(idx, wd, keep, recent, ids, bounds, counts, lens, sd, sn, st);
        return true;
    });
}

// Whether every row that an eviction may write lies in the destination (both are caches of four dimensions).
bool holds_rows(const at::Tensor& K, const at::Tensor& K_to, const Room& room, bool in4) {
    const int64_t B = room.known ? room.B() : K.size(0), H = room.known ? room.H() : K.size(1), rows = room.known ? room.tokens() : K.size(2);
    if (K.size(0) < B || K.size(1) < H || K_to.size(0) < B || K_to.size(1) < H || K_to.size(2) < rows || K.size(3) != K_to.size(3) ||
        (!in4 && K.size(3) != LC_HEAD_DIM)) {
        PyErr_SetString(PyExc_AssertionError, "K_to and V_to must have room for the index's sequences, heads and max_tokens rows like K's");
        return false;
    }
    return true;
}

// evict_rows(handle, keep_ids, keep_bounds, keep_counts, K, V, K_to, V_to, weights, weights_to, stream, room)
PyObject* evict_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n);
    if (!a.count(12)) return nullptr;
    return guarded(a, [&](int* rc) {
        const at::Tensor *K = a.tensor(4), *V = a.tensor(5), *K_to = a.tensor(6), *V_to = a.tensor(7);
        if (!K || !V || !K_to || !V_to || a.foreign()) return false;
        const bool in4 = K->element_size() == 1;
        int64_t s[3], st_to[3];
        for (const at::Tensor* t : {K, V, K_to, V_to})
            if (t->element_size() != (in4 ? 1 : 2)) return false;
        if (in4 ? !cache4_strides(*K, *V, s) || !cache4_strides(*K_to, *V_to, st_to) : !cache_strides(*K, *V, true, s) || !cache_strides(*K_to, *V_to, true, st_to))
            return true;
        const at::Tensor *ids_t = a.tensor(1), *bounds_t = a.tensor(2), *n_t = a.tensor(3), *w_t = a.tensor(8), *w_to_t = a.tensor(9);
        const Room room = a.room(11);
        if (!holds_rows(*K, *K_to, room, in4) || !keep_tables(room, ids_t, bounds_t, n_t)) return true;
        const int64_t pairs = room.B() * room.H();
        if (room.known && (!table(w_t, true, pairs, room.chunks(), "weights") || !table(w_to_t, true, pairs, room.chunks(), "weights_to"))) return true;
        const int32_t* const ids = static_cast<const int32_t*>(a.ptr(1));
        const int32_t* const bounds = static_cast<const int32_t*>(a.ptr(2));
        const int32_t* const counts = static_cast<const int32_t*>(a.ptr(3));
        const float* const w = static_cast<const float*>(a.ptr(8));
        float* const w_to = static_cast<float*>(a.ptr(9));
        if (a.foreign()) return false;
        void* const st = a.stream(10);
        if (PyErr_Occurred()) return false;
        lc_index* const idx = a.handle(0);
        if (PyErr_Occurred()) return false;
        const void *kd = K->data_ptr(), *vd = V->data_ptr();
        void *kt = K_to->data_ptr(), *vt = V_to->data_ptr();
        const Unlocked unlocked;
        *rc = (in4 ? g_evict_rows4 : g_evict_rows)(idx, ids, bounds, counts, kd, vd, s, kt, vt, st_to, w, w_to, st);
        return true;
    });
}

template <typename F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", fast(bind), METH_FASTCALL, "addresses of the library's entry points"},
    {"decode_step", fast(decode_step), METH_FASTCALL, ""},
    {"retrieve", fast(retrieve), METH_FASTCALL, ""},
    {"sparse_decode", fast(sparse_decode), METH_FASTCALL, ""},
    {"append", fast(append), METH_FASTCALL, ""},
    {"bind4", fast(bind4), METH_FASTCALL, "addresses of the 4-bit cache's and the eviction's entry points"},
    {"move4", fast(move4), METH_FASTCALL, ""},
    {"sparse_decode4", fast(sparse_decode4), METH_FASTCALL, ""},
    {"append4", fast(append4), METH_FASTCALL, ""},
    {"weigh_chunks", fast(weigh_chunks), METH_FASTCALL, ""},
    {"evict_select", fast(evict_select), METH_FASTCALL, ""},
    {"evict_rows", fast(evict_rows), METH_FASTCALL, ""},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lychee_torch", "Tensor marshalling of the per-token entry points.", -1,
                      methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lychee_torch() { return PyModule_Create(&module); }
