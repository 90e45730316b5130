// The hot entry points of the Python binding without Python in between: a small call took 2.5 us of attribute look-ups on
// its tensors before it reached the library, of the 6 that it took in all, and the smallest kernels take 4.
//
// Each function here takes exactly what the Python function of its name takes, by position.  It answers only the plain
// case (exact torch tensors of the right type and layout, ints and floats) with the library's status; for everything
// else, also for whatever is wrong, it returns None, and the Python function does the whole call itself, with its own
// checks and messages.
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "../../include/chipmunk.h"

namespace {

struct Entry {
    const char* name;
    void* at;
};
Entry entries[] = {{"chipmunk_voxel_reorder", nullptr},       {"chipmunk_topk_cols", nullptr},
                   {"chipmunk_attn_sparse_delta", nullptr},   {"chipmunk_attn_dense", nullptr},
                   {"chipmunk_attn_dense_colsum_stale", nullptr}, {"chipmunk_mlp_tile_mean_preact", nullptr},
                   {"chipmunk_mlp_sparse_delta", nullptr},    {"chipmunk_mlp_dense", nullptr},
                   {"chipmunk_linear", nullptr},              {"chipmunk_rope", nullptr},
                   {"chipmunk_attn_packed", nullptr},         {"chipmunk_norm_rope", nullptr},
                   {"chipmunk_cache_write", nullptr},         {"chipmunk_cache_read", nullptr},
                   {"chipmunk_attn_paged", nullptr},          {"chipmunk_norm_rope_grad", nullptr}};
enum { kReorder, kTopk, kAttnDelta, kAttnDense, kAttnRefresh, kScores, kMlpDelta, kMlpDense, kLinear, kRope, kAttnPacked, kNormRope, kCacheWrite, kCacheRead, kAttnPaged, kNormRopeGrad };
PyObject* current_device = nullptr;   // torch's functions that name the current device and, for a device, its current stream
PyObject* raw_stream = nullptr;

// One call's arguments; ok turns false with the first that the plain case does not cover.
struct Args {
    PyObject* const* v;
    bool ok;

    const at::Tensor* tensor(int i) {
        if (!ok || !THPVariable_CheckExact(v[i])) {
            ok = false;
            return nullptr;
        }
        return &THPVariable_Unpack(v[i]);
    }
    // data of a contiguous GPU tensor of this type; None: null
    void* data(int i, at::ScalarType type) {
        if (!ok || none(i)) return nullptr;
        const at::Tensor* t = tensor(i);
        if (!ok || t->scalar_type() != type || !t->is_cuda() || !t->is_contiguous()) {
            ok = false;
            return nullptr;
        }
        return t->data_ptr();
    }
    const uint16_t* bf16(int i) { return static_cast<const uint16_t*>(data(i, at::kBFloat16)); }
    uint16_t* bf16_out(int i) { return static_cast<uint16_t*>(data(i, at::kBFloat16)); }
    int32_t* i32(int i) { return static_cast<int32_t*>(data(i, at::kInt)); }
    float* f32(int i) { return static_cast<float*>(data(i, at::kFloat)); }
    // size `dim` of a tensor of `dims` dimensions (-1: the last of any)
    int size(int i, int dims, int dim) {
        const at::Tensor* t = tensor(i);
        if (!ok || (dims >= 0 ? t->dim() != dims : t->dim() < 1)) {
            ok = false;
            return 0;
        }
        const int64_t n = t->size(dims >= 0 ? dim : t->dim() - 1);
        if (n > INT_MAX) ok = false;
        return (int)n;
    }
    bool none(int i) const { return v[i] == Py_None; }
    int rows(int i) {          // a tensor's first size
        const at::Tensor* t = tensor(i);
        if (!ok || t->dim() < 1 || t->size(0) > INT_MAX) {
            ok = false;
            return 0;
        }
        return (int)t->size(0);
    }
    size_t elements(int i) {   // None: 0
        if (!ok || none(i)) return 0;
        const at::Tensor* t = tensor(i);
        return ok ? (size_t)t->numel() : 0;
    }
    int integer(int i) {
        if (!ok || !PyLong_CheckExact(v[i])) {
            ok = false;
            return 0;
        }
        int over = 0;
        const long n = PyLong_AsLongAndOverflow(v[i], &over);
        if (over || n > INT_MAX || n < INT_MIN) ok = false;
        return (int)n;
    }
    float real(int i) {
        if (!ok || !PyFloat_CheckExact(v[i])) {
            ok = false;
            return 0.f;
        }
        return (float)PyFloat_AS_DOUBLE(v[i]);
    }
    void* stream() {
        if (!ok) return nullptr;
        PyObject* device = PyObject_CallNoArgs(current_device);
        PyObject* s = device ? PyObject_CallOneArg(raw_stream, device) : nullptr;
        void* at = s ? PyLong_AsVoidPtr(s) : nullptr;
        Py_XDECREF(device);
        Py_XDECREF(s);
        if (PyErr_Occurred()) ok = false;
        return at;
    }
};

// call(a): the library's status, the GIL released around the library itself by `run`, whose first argument only names the
// function's type (a reference to the function itself would need the library at link time)
template <typename Call>
PyObject* answer(int entry, PyObject* const* args, Py_ssize_t n, Py_ssize_t want, Call&& call) {
    if (!entries[entry].at || n != want) Py_RETURN_NONE;
    Args a{args, true};
    int32_t status = 0;
    try {
        call(a, [&](auto f, auto... values) {
            if (!a.ok) return;
            PyThreadState* state = PyEval_SaveThread();
            status = reinterpret_cast<decltype(f)>(entries[entry].at)(values...);
            PyEval_RestoreThread(state);
        });
    } catch (...) {
        a.ok = false;
    }
    if (!a.ok) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}

// Arguments are read into variables, in order, before the call: a call's own arguments have no order, and `ok` must be
// known.

// src, dst, perm, inv_perm, n_prefix, T, H, W, n_suffix, vt, vh, vw, inverse
PyObject* voxel_reorder(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kReorder, args, n, 13, [](Args& a, auto run) {
        const at::Tensor *src = a.tensor(0), *dst = a.tensor(1);   // (permutations alone: the Python function)
        if (!a.ok || src->dim() < 2 || src->size(0) < 1 || src->size(1) < 1 || src->sizes() != dst->sizes() || src->size(0) > INT_MAX) {
            a.ok = false;
            return;
        }
        const int64_t row = src->numel() / (src->size(0) * src->size(1)) * (int64_t)src->element_size();
        if (row > INT_MAX || !PyBool_Check(a.v[12])) a.ok = false;
        const void* from = a.data(0, src->scalar_type());
        void* to = a.data(1, src->scalar_type());
        int32_t *perm = a.i32(2), *inv = a.i32(3);
        int g[8];
        for (int i = 0; i < 8; i++) g[i] = a.integer(4 + i);
        void* s = a.stream();
        run(decltype(&chipmunk_voxel_reorder){}, from, to, perm, inv, (int)src->size(0), g[0], g[1], g[2], g[3], g[4], g[5], g[6], g[7], (int)row,
            (int)(a.v[12] == Py_True), s);
    });
}

// cur, prev, k, idx, counts
PyObject* topk_cols(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kTopk, args, n, 5, [](Args& a, auto run) {
        auto rows = [&](int i) -> const at::Tensor* {   // dense rows that a leading dimension may space
            const at::Tensor* t = a.tensor(i);
            if (a.ok && (t->dim() != 2 || t->scalar_type() != at::kFloat || !t->is_cuda() || (t->size(1) > 1 && t->stride(1) != 1))) a.ok = false;
            return t;
        };
        const at::Tensor* cur = rows(0);
        const at::Tensor* prev = a.none(1) ? nullptr : rows(1);
        if (!a.ok || (prev && (prev->sizes() != cur->sizes() || prev->stride(0) != cur->stride(0))) || cur->size(0) > INT_MAX || cur->size(1) > INT_MAX) {
            a.ok = false;
            return;
        }
        const int k = a.integer(2);
        int32_t *idx = a.i32(3), *counts = a.i32(4);
        const int k_stride = a.size(3, -1, 0);
        void* s = a.stream();
        run(decltype(&chipmunk_topk_cols){}, (const float*)cur->data_ptr(), prev ? (const float*)prev->data_ptr() : nullptr, (int)cur->size(0), (int)cur->size(1),
            (int64_t)cur->stride(0), k, idx, counts, k_stride, s);
    });
}

// q, k, v, idx, counts, base, out, c, softmax_scale, o_scale
PyObject* attn_sparse_delta(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kAttnDelta, args, n, 10, [](Args& a, auto run) {
        const uint16_t *q = a.bf16(0), *k = a.bf16(1), *v = a.bf16(2);
        const int B = a.size(0, 4, 0), H = a.size(0, 4, 1), N = a.size(0, 4, 2), E = a.size(0, 4, 3);
        const int32_t *idx = a.i32(3), *counts = a.i32(4);
        const int k_stride = a.none(3) ? 0 : a.size(3, -1, 0);
        const uint16_t* base = a.bf16(5);
        uint16_t* out = a.bf16_out(6);
        const int c = a.integer(7);
        const float scale = a.real(8), o_scale = a.real(9);
        void* s = a.stream();
        run(decltype(&chipmunk_attn_sparse_delta){}, q, k, v, idx, counts, base, out, B, H, N, E, c, k_stride, scale, o_scale, s);
    });
}

// q, k, v, out, colsum, c, softmax_scale, ws
PyObject* attn_dense(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kAttnDense, args, n, 8, [](Args& a, auto run) {
        const uint16_t *q = a.bf16(0), *k = a.bf16(1), *v = a.bf16(2);
        const int B = a.size(0, 4, 0), H = a.size(0, 4, 1), N = a.size(0, 4, 2), E = a.size(0, 4, 3);
        uint16_t* out = a.bf16_out(3);
        float* colsum = a.f32(4);
        const int64_t ld = a.none(4) ? 0 : a.size(4, -1, 0);
        const int c = a.integer(5);
        const float scale = a.real(6);
        void* ws = a.data(7, at::kByte);
        const size_t bytes = a.elements(7);
        void* s = a.stream();
        run(decltype(&chipmunk_attn_dense){}, q, k, v, out, colsum, ld, B, H, N, E, c, scale, ws, bytes, s);
    });
}

// q, k, v, out, prev_m, prev_l, colsum, c, softmax_scale, new_m, new_l
PyObject* attn_dense_colsum_stale(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kAttnRefresh, args, n, 11, [](Args& a, auto run) {
        const uint16_t *q = a.bf16(0), *k = a.bf16(1), *v = a.bf16(2);
        const int B = a.size(0, 4, 0), H = a.size(0, 4, 1), N = a.size(0, 4, 2), E = a.size(0, 4, 3);
        uint16_t* out = a.bf16_out(3);
        const float *prev_m = a.f32(4), *prev_l = a.f32(5);
        float* colsum = a.f32(6);
        const int64_t ld = a.size(6, -1, 0);
        const int c = a.integer(7);
        const float scale = a.real(8);
        float *new_m = a.f32(9), *new_l = a.f32(10);
        void* s = a.stream();
        run(decltype(&chipmunk_attn_dense_colsum_stale){}, q, k, v, out, prev_m, prev_l, colsum, ld, new_m, new_l, B, H, N, E, c, scale, s);
    });
}

// x, w1, T, c, ws
PyObject* mlp_tile_mean_preact(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kScores, args, n, 5, [](Args& a, auto run) {
        const uint16_t *x = a.bf16(0), *w1 = a.bf16(1);
        const int B = a.size(0, 3, 0), N = a.size(0, 3, 1), D = a.size(0, 3, 2), F = a.rows(1);
        float* T = a.f32(2);
        const int c = a.integer(3);
        void* ws = a.data(4, at::kByte);
        const size_t bytes = a.elements(4);
        void* s = a.stream();
        run(decltype(&chipmunk_mlp_tile_mean_preact){}, x, w1, T, B, N, D, F, c, ws, bytes, s);
    });
}

// x, w1, b1, w2, idx, counts, a_cache, o_cache, c, act, ws
PyObject* mlp_sparse_delta(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kMlpDelta, args, n, 11, [](Args& a, auto run) {
        const uint16_t *x = a.bf16(0), *w1 = a.bf16(1), *b1 = a.bf16(2), *w2 = a.bf16(3);
        const int B = a.size(0, 3, 0), N = a.size(0, 3, 1), D = a.size(0, 3, 2), F = a.rows(1);
        const int32_t *idx = a.i32(4), *counts = a.i32(5);
        const int k_stride = a.size(4, -1, 0);
        uint16_t *a_cache = a.bf16_out(6), *o_cache = a.bf16_out(7);
        const int64_t a_ld = a.size(6, -1, 0);
        const int c = a.integer(8), act = a.integer(9);
        void* ws = a.data(10, at::kByte);
        const size_t bytes = a.elements(10);
        void* s = a.stream();
        run(decltype(&chipmunk_mlp_sparse_delta){}, x, w1, b1, w2, idx, counts, a_cache, a_ld, o_cache, B, N, D, F, c, k_stride, act, ws, bytes, s);
    });
}

// x, w1, b1, w2, b2, out, a_cache, c, act
PyObject* mlp_dense(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kMlpDense, args, n, 9, [](Args& a, auto run) {
        const uint16_t *x = a.bf16(0), *w1 = a.bf16(1), *b1 = a.bf16(2), *w2 = a.bf16(3), *b2 = a.bf16(4);
        const int B = a.size(0, 3, 0), N = a.size(0, 3, 1), D = a.size(0, 3, 2), F = a.rows(1);
        uint16_t *out = a.bf16_out(5), *a_cache = a.bf16_out(6);
        const int64_t a_ld = a.size(6, -1, 0);
        const int c = a.integer(7), act = a.integer(8);
        void* s = a.stream();
        run(decltype(&chipmunk_mlp_dense){}, x, w1, b1, w2, b2, out, a_cache, a_ld, B, N, D, F, c, act, s);
    });
}

// ---- tensors with strides: one call's are on the current device, of one element type, with dense last dimensions ----
struct Strided {
    Args& a;
    int device = -1;
    at::ScalarType element = at::kBFloat16;

    // the call's element type is that of argument i
    explicit Strided(Args& args, int i) : a(args) {
        const at::Tensor* t = a.tensor(i);
        if (!a.ok) return;
        element = t->scalar_type();
        if (element != at::kBFloat16 && element != at::kHalf) a.ok = false;
        PyObject* number = PyObject_CallNoArgs(current_device);
        device = number ? (int)PyLong_AsLong(number) : -1;
        Py_XDECREF(number);
        if (PyErr_Occurred()) a.ok = false;
    }
    const at::Tensor* tensor(int i, int dims, at::ScalarType type) {
        const at::Tensor* t = a.tensor(i);
        if (!a.ok) return nullptr;
        if (t->dim() != dims || t->scalar_type() != type || t->numel() == 0 || t->device().type() != at::kCUDA || t->device().index() != device ||
            (t->size(dims - 1) > 1 && t->stride(dims - 1) != 1))
            a.ok = false;
        for (int d = 0; a.ok && d < dims; d++)
            if (t->size(d) > INT_MAX) a.ok = false;
        return a.ok ? t : nullptr;
    }
    const at::Tensor* elements(int i, int dims) { return tensor(i, dims, element); }
    const at::Tensor* optional(int i, int dims, at::ScalarType type) { return a.ok && !a.none(i) ? tensor(i, dims, type) : nullptr; }
    int number() const { return element == at::kBFloat16 ? 0 : 1; }
    bool truth(int i) {
        if (a.ok && !PyBool_Check(a.v[i])) a.ok = false;
        return a.ok && a.v[i] == Py_True;
    }
};
const uint16_t* elements_of(const at::Tensor* t) { return t ? static_cast<const uint16_t*>(t->data_ptr()) : nullptr; }

// x, w, bias, residual, out, act
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kLinear, args, n, 6, [](Args& a, auto run) {
        Strided s(a, 0);
        const at::Tensor *x = s.elements(0, 2), *w = s.elements(1, 2), *bias = s.optional(2, 1, s.element), *residual = s.optional(3, 2, s.element), *out = s.elements(4, 2);
        const int act = a.integer(5);
        if (!a.ok || !w->is_contiguous() || w->size(1) != x->size(1) || out->size(0) != x->size(0) || out->size(1) != w->size(0) ||
            (residual && residual->sizes() != out->sizes()) || (bias && bias->size(0) != w->size(0))) {
            a.ok = false;
            return;
        }
        void* stream = a.stream();
        run(decltype(&chipmunk_linear){}, elements_of(x), x->stride(0), elements_of(w), elements_of(bias), elements_of(residual), residual ? residual->stride(0) : (int64_t)0,
            const_cast<uint16_t*>(elements_of(out)), out->stride(0), (int)x->size(0), (int)x->size(1), (int)w->size(0), act, s.number(), stream);
    });
}

// x, pos, freqs, out, axes, halves, inverse
PyObject* rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kRope, args, n, 7, [](Args& a, auto run) {
        Strided s(a, 0);
        const at::Tensor *x = s.elements(0, 3), *pos = s.tensor(1, 2, at::kInt), *freqs = s.tensor(2, 1, at::kDouble), *out = s.elements(3, 3);
        if (!a.ok || (!PyList_CheckExact(a.v[4]) && !PyTuple_CheckExact(a.v[4])) || PySequence_Fast_GET_SIZE(a.v[4]) != 3) {
            a.ok = false;
            return;
        }
        Args axes{PySequence_Fast_ITEMS(a.v[4]), true};
        const int t = axes.integer(0), h = axes.integer(1), w = axes.integer(2);
        const bool halves = s.truth(5), inverse = s.truth(6);
        if (!a.ok || !axes.ok || out->sizes() != x->sizes() || pos->size(0) != x->size(0) || pos->size(1) != 3 || !pos->is_contiguous() ||
            freqs->size(0) != (int64_t)t + h + w) {
            a.ok = false;
            return;
        }
        void* stream = a.stream();
        run(decltype(&chipmunk_rope){}, elements_of(x), x->stride(0), x->stride(1), (const int32_t*)pos->data_ptr(), (const double*)freqs->data_ptr(),
            const_cast<uint16_t*>(elements_of(out)), out->stride(0), out->stride(1), (int)x->size(0), (int)x->size(1), (int)x->size(2), t, h, w, (int)halves, (int)inverse,
            s.number(), stream);
    });
}

// q, k, v, cu_q, cu_k, out, max_q, max_k, causal, softmax_scale, k_len, ws
PyObject* attn_packed(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kAttnPacked, args, n, 12, [](Args& a, auto run) {
        Strided s(a, 0);
        const at::Tensor *q = s.elements(0, 3), *k = s.elements(1, 3), *v = s.elements(2, 3), *cu_q = s.tensor(3, 1, at::kInt), *cu_k = s.tensor(4, 1, at::kInt),
                         *out = s.elements(5, 3), *k_len = s.optional(10, 1, at::kInt), *ws = s.optional(11, 1, at::kByte);
        const int max_q = a.integer(6), max_k = a.integer(7);
        const bool causal = s.truth(8);
        const float scale = a.real(9);
        if (!a.ok || out->sizes() != q->sizes() || k->sizes() != v->sizes() || k->size(2) != q->size(2) || cu_k->size(0) != cu_q->size(0) ||
            (k_len && k_len->size(0) != cu_q->size(0) - 1)) {
            a.ok = false;
            return;
        }
        void* stream = a.stream();
        run(decltype(&chipmunk_attn_packed){}, elements_of(q), q->stride(0), q->stride(1), elements_of(k), k->stride(0), k->stride(1), elements_of(v), v->stride(0), v->stride(1),
            const_cast<uint16_t*>(elements_of(out)), out->stride(0), out->stride(1), (const int32_t*)cu_q->data_ptr(), (const int32_t*)cu_k->data_ptr(),
            k_len ? (const int32_t*)k_len->data_ptr() : nullptr, (int)(cu_q->size(0) - 1), (int)q->size(0), (int)k->size(0), (int)q->size(1), (int)k->size(1), (int)q->size(2), max_q,
            max_k, (int)causal, scale, s.number(), ws ? ws->data_ptr() : nullptr, ws ? (size_t)ws->numel() : (size_t)0, stream);
    });
}

// Three sizes in a list or a tuple
struct Axes {
    int t = 0, h = 0, w = 0;
    Axes(Args& a, int i) {
        if (!a.ok || (!PyList_CheckExact(a.v[i]) && !PyTuple_CheckExact(a.v[i])) || PySequence_Fast_GET_SIZE(a.v[i]) != 3) {
            a.ok = false;
            return;
        }
        Args axes{PySequence_Fast_ITEMS(a.v[i]), true};
        t = axes.integer(0), h = axes.integer(1), w = axes.integer(2);
        a.ok = axes.ok;
    }
    int64_t pairs() const { return (int64_t)t + h + w; }
};

// x, q_weight, k_weight, q_heads, pos, freqs, out, axes, eps, halves
PyObject* norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kNormRope, args, n, 10, [](Args& a, auto run) {
        Strided s(a, 0);
        const at::Tensor *x = s.elements(0, 3), *wq = s.optional(1, 1, s.element), *wk = s.optional(2, 1, s.element), *pos = s.optional(4, 2, at::kInt),
                         *freqs = s.optional(5, 1, at::kDouble), *out = s.elements(6, 3);
        const int q_heads = a.integer(3);
        const Axes axes(a, 7);
        const float eps = a.real(8);
        const bool halves = s.truth(9);
        if (!a.ok || out->sizes() != x->sizes() || (wq && wq->size(0) != x->size(2)) || (wk && wk->size(0) != x->size(2)) ||
            (pos && (pos->size(0) != x->size(0) || pos->size(1) != 3 || !pos->is_contiguous())) || (freqs && freqs->size(0) != axes.pairs())) {
            a.ok = false;
            return;
        }
        void* stream = a.stream();
        run(decltype(&chipmunk_norm_rope){}, elements_of(x), x->stride(0), x->stride(1), elements_of(wq), elements_of(wk), q_heads, pos ? (const int32_t*)pos->data_ptr() : nullptr,
            freqs ? (const double*)freqs->data_ptr() : nullptr, const_cast<uint16_t*>(elements_of(out)), out->stride(0), out->stride(1), (int)x->size(0), (int)x->size(1),
            (int)x->size(2), axes.t, axes.h, axes.w, eps, (int)halves, s.number(), stream);
    });
}

// grad, x, q_weight, k_weight, q_heads, pos, freqs, dx, dq_weight, dk_weight, axes, eps, halves, ws
PyObject* norm_rope_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kNormRopeGrad, args, n, 14, [](Args& a, auto run) {
        Strided s(a, 1);
        const at::Tensor *grad = s.elements(0, 3), *x = s.elements(1, 3), *wq = s.optional(2, 1, s.element), *wk = s.optional(3, 1, s.element), *pos = s.optional(5, 2, at::kInt),
                         *freqs = s.optional(6, 1, at::kDouble), *dx = s.elements(7, 3), *dq = s.optional(8, 1, at::kFloat), *dk = s.optional(9, 1, at::kFloat),
                         *ws = s.optional(13, 1, at::kByte);
        const int q_heads = a.integer(4);
        const Axes axes(a, 10);
        const float eps = a.real(11);
        const bool halves = s.truth(12);
        if (!a.ok || dx->sizes() != x->sizes() || grad->sizes() != x->sizes() || (wq && wq->size(0) != x->size(2)) || (wk && wk->size(0) != x->size(2)) ||
            (dq && dq->size(0) != x->size(2)) || (dk && dk->size(0) != x->size(2)) || (pos && (pos->size(0) != x->size(0) || pos->size(1) != 3 || !pos->is_contiguous())) ||
            (freqs && freqs->size(0) != axes.pairs())) {
            a.ok = false;
            return;
        }
        void* stream = a.stream();
        run(decltype(&chipmunk_norm_rope_grad){}, elements_of(grad), grad->stride(0), grad->stride(1), elements_of(x), x->stride(0), x->stride(1), elements_of(wq), elements_of(wk),
            q_heads, pos ? (const int32_t*)pos->data_ptr() : nullptr, freqs ? (const double*)freqs->data_ptr() : nullptr, const_cast<uint16_t*>(elements_of(dx)), dx->stride(0),
            dx->stride(1), dq ? (float*)dq->data_ptr() : nullptr, dk ? (float*)dk->data_ptr() : nullptr, (int)x->size(0), (int)x->size(1), (int)x->size(2), axes.t, axes.h, axes.w,
            eps, (int)halves, s.number(), ws ? ws->data_ptr() : nullptr, ws ? (size_t)ws->numel() : (size_t)0, stream);
    });
}

// What a Pages object says of itself: the address of its struct, its device, heads and E
struct PagesArg {
    const chipmunk_pages* at = nullptr;
    int heads = 0, E = 0;
    PagesArg(Strided& s, int i) {
        Args& a = s.a;
        if (!a.ok || !PyTuple_CheckExact(a.v[i]) || PyTuple_GET_SIZE(a.v[i]) != 4) {
            a.ok = false;
            return;
        }
        at = static_cast<const chipmunk_pages*>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(a.v[i], 0)));
        Args rest{PySequence_Fast_ITEMS(a.v[i]), true};
        const int device = rest.integer(1);
        heads = rest.integer(2), E = rest.integer(3);
        if (PyErr_Occurred() || !rest.ok || !at || device != s.device) a.ok = false;
    }
};

// k, v, rows, pages (writing) or pages, rows, k, v (reading)
template <class Run>
void cache_call(Args& a, int k_at, int v_at, int rows_at, int pages_at, Run&& run) {
    Strided s(a, k_at);
    const at::Tensor *k = s.elements(k_at, 3), *v = s.elements(v_at, 3), *rows = s.tensor(rows_at, 1, at::kLong);
    const PagesArg pages(s, pages_at);
    if (!a.ok || v->sizes() != k->sizes() || rows->size(0) != k->size(0) || k->size(1) != pages.heads || k->size(2) != pages.E) {
        a.ok = false;
        return;
    }
    run(s, k, v, (const int64_t*)rows->data_ptr(), pages.at, a.stream());
}
PyObject* cache_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kCacheWrite, args, n, 4, [](Args& a, auto run) {
        cache_call(a, 0, 1, 2, 3, [&](Strided& s, const at::Tensor* k, const at::Tensor* v, const int64_t* rows, const chipmunk_pages* pages, void* stream) {
            run(decltype(&chipmunk_cache_write){}, elements_of(k), k->stride(0), k->stride(1), elements_of(v), v->stride(0), v->stride(1), rows, pages, (int)k->size(0), s.number(), stream);
        });
    });
}
PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kCacheRead, args, n, 4, [](Args& a, auto run) {
        cache_call(a, 2, 3, 1, 0, [&](Strided& s, const at::Tensor* k, const at::Tensor* v, const int64_t* rows, const chipmunk_pages* pages, void* stream) {
            run(decltype(&chipmunk_cache_read){}, pages, rows, const_cast<uint16_t*>(elements_of(k)), k->stride(0), k->stride(1), const_cast<uint16_t*>(elements_of(v)), v->stride(0),
                v->stride(1), (int)k->size(0), s.number(), stream);
        });
    });
}

// q, pages, table, cu_q, k_len, out, max_q, max_k, causal, softmax_scale, window, sinks, ws
PyObject* attn_paged(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return answer(kAttnPaged, args, n, 13, [](Args& a, auto run) {
        Strided s(a, 0);
        const at::Tensor *q = s.elements(0, 3), *table = s.tensor(2, 2, at::kInt), *cu_q = s.tensor(3, 1, at::kInt), *k_len = s.tensor(4, 1, at::kInt), *out = s.elements(5, 3),
                         *ws = s.optional(12, 1, at::kByte);
        const PagesArg pages(s, 1);
        const int max_q = a.integer(6), max_k = a.integer(7), window = a.integer(10), sinks = a.integer(11);
        const bool causal = s.truth(8);
        const float scale = a.real(9);
        if (!a.ok || out->sizes() != q->sizes() || q->size(2) != pages.E || cu_q->size(0) != k_len->size(0) + 1 || table->size(0) != k_len->size(0)) {
            a.ok = false;
            return;
        }
        void* stream = a.stream();
        run(decltype(&chipmunk_attn_paged){}, elements_of(q), q->stride(0), q->stride(1), pages.at, (const int32_t*)table->data_ptr(), table->stride(0), (int)table->size(1),
            const_cast<uint16_t*>(elements_of(out)), out->stride(0), out->stride(1), (const int32_t*)cu_q->data_ptr(), (const int32_t*)k_len->data_ptr(), (int)k_len->size(0),
            (int)q->size(0), (int)q->size(1), max_q, max_k, (int)causal, window, sinks, scale, s.number(), ws ? ws->data_ptr() : nullptr, ws ? (size_t)ws->numel() : (size_t)0, stream);
    });
}

// bind(addresses: dict of names, current_device, raw_stream)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 3 || !PyDict_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "bind(addresses, current_device, raw_stream)");
        return nullptr;
    }
    for (Entry& e : entries) {
        PyObject* at = PyDict_GetItemString(args[0], e.name);
        e.at = at ? PyLong_AsVoidPtr(at) : nullptr;
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(args[1]);
    Py_XSETREF(current_device, args[1]);
    Py_INCREF(args[2]);
    Py_XSETREF(raw_stream, args[2]);
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind), FAST(voxel_reorder), FAST(topk_cols), FAST(attn_sparse_delta), FAST(attn_dense),
                         FAST(attn_dense_colsum_stale), FAST(mlp_tile_mean_preact), FAST(mlp_sparse_delta), FAST(mlp_dense),
                         FAST(linear), FAST(rope), FAST(attn_packed), FAST(norm_rope), FAST(cache_write), FAST(cache_read), FAST(attn_paged), FAST(norm_rope_grad),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The stamp names the torch, the Python and the header that this was compiled with.  It is looked for in the file before
// the file is loaded.
PyMODINIT_FUNC PyInit__native() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", CHIPMUNK_BINDING_STAMP) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
