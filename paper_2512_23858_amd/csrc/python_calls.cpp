// Native argument marshalling of the Python package: one C function per launching call.  Each takes the Shape object and
// torch tensors (or None) by position, checks device, layout and element type, and hands raw pointers and the current
// stream to the C ABI.  It returns the C ABI's status, or kCheckFailed when an argument does not pass; the Python side then
// runs its own checks, which raise the matching exception.
//
// Host time per call matters: a short verification step is made of calls whose kernels take a few microseconds, and the
// stream runs dry when the host cannot enqueue that fast.  Marshalling through ctypes took 6-7 us per call beside two
// launches of 3-4 us each; this takes well under one.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "ygg.h"

namespace {

constexpr long kCheckFailed = -1;

PyObject* g_field[12];
const char* const kField[12] = {"batch", "n_q_heads", "n_kv_heads", "head_dim", "depth", "width", "n_nodes", "vocab",
                                "kv_dtype", "softmax_scale", "kv_capacity", "max_seq_len"};

PyObject* attribute(PyObject* o, int i) {   // new reference
    PyObject** d = _PyObject_GetDictPtr(o);
    if (d && *d)
        if (PyObject* v = PyDict_GetItemWithError(*d, g_field[i])) {   // the usual case: an instance's own field
            Py_INCREF(v);
            return v;
        }
    PyErr_Clear();
    return PyObject_GetAttr(o, g_field[i]);
}

bool read_int(PyObject* o, int i, int64_t lo, int64_t hi, int64_t& out) {
    PyObject* v = attribute(o, i);
    if (!v) return false;
    out = PyLong_AsLongLong(v);
    Py_DECREF(v);
    return !(out == -1 && PyErr_Occurred()) && out >= lo && out <= hi;
}

// False (no exception set) if a field is missing, not a number or out of the C type's range.
bool read_shape(PyObject* o, ygg_shape& s) {
    int32_t* const dst[12] = {&s.batch, &s.n_q_heads, &s.n_kv_heads, &s.head_dim, &s.depth, &s.width, &s.n_nodes, &s.vocab,
                              &s.kv_dtype, nullptr, nullptr, &s.max_seq_len};
    bool ok = true;
    for (int i = 0; i < 12 && ok; ++i) {
        int64_t v = 0;
        if (i == 9) {
            PyObject* f = attribute(o, i);
            const double x = f ? PyFloat_AsDouble(f) : -1.0;
            Py_XDECREF(f);
            ok = !PyErr_Occurred();
            s.softmax_scale = (float)x;
        } else if (i == 10) {
            ok = read_int(o, i, INT64_MIN, INT64_MAX, s.kv_capacity);
        } else if ((ok = read_int(o, i, INT32_MIN, INT32_MAX, v))) {
            *dst[i] = (int32_t)v;
        }
    }
    PyErr_Clear();
    return ok;
}

// The tensor arguments of one call: pointers come out in order, and one failed check marks the call.
struct Args {
    PyObject* const* a;
    bool ok = true;
    void* ptr(int i, at::ScalarType want, bool any = false) {
        PyObject* o = a[i];
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous() || (!any && t.scalar_type() != want)) { ok = false; return nullptr; }
        return t.data_ptr();
    }
    template <typename T> T* typed(int i, at::ScalarType want) { return static_cast<T*>(ptr(i, want)); }
    int32_t* ints(int i) { return typed<int32_t>(i, at::kInt); }
    float* floats(int i) { return typed<float>(i, at::kFloat); }
    void* scratch(int i, size_t& bytes) {
        void* p = ptr(i, at::kByte, true);
        bytes = p ? THPVariable_Unpack(a[i]).nbytes() : 0;
        return p;
    }
    // A tensor [B, N, ..] whose trailing dimensions are dense and whose B * N rows lie evenly, each behind the one before: the row
    // stride in elements (an expanded tensor's stride of 0 would be the calls' word for dense rows, which it does not have)
    void* rows(int i, at::ScalarType want, int64_t& stride, bool any = false) {
        PyObject* o = a[i];
        stride = 0;
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.dim() < 3 || (!any && t.scalar_type() != want)) { ok = false; return nullptr; }
        int64_t inner = 1;
        for (int64_t d = t.dim() - 1; d >= 2; --d) {
            if (t.size(d) > 1 && t.stride(d) != inner) { ok = false; return nullptr; }
            inner *= t.size(d);
        }
        const int64_t B = t.size(0), N = t.size(1);
        stride = N > 1 ? t.stride(1) : B > 1 ? t.stride(0) : inner;
        if ((B > 1 && N > 1 && t.stride(0) != N * stride) || ((B > 1 || N > 1) && stride < inner)) { ok = false; return nullptr; }
        return t.data_ptr();
    }
    // A tensor [N, ..] of rows likewise
    void* flat_rows(int i, at::ScalarType want, int64_t& stride) {
        PyObject* o = a[i];
        stride = 0;
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.dim() < 2 || t.scalar_type() != want) { ok = false; return nullptr; }
        int64_t inner = 1;
        for (int64_t d = t.dim() - 1; d >= 1; --d) {
            if (t.size(d) > 1 && t.stride(d) != inner) { ok = false; return nullptr; }
            inner *= t.size(d);
        }
        stride = t.size(0) > 1 ? t.stride(0) : inner;
        if (stride < inner) { ok = false; return nullptr; }
        return t.data_ptr();
    }
    // A given tensor has `per` elements to a sequence (the kernels go by the shape, not by the tensors).  More sequences may follow,
    // and a single one may be longer: where several are, the next one would not begin where the kernels step to.
    void holds(int i, int64_t seqs, int64_t per) {
        if (!ok || a[i] == Py_None) return;
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        const int64_t n = t.numel();
        ok = n == seqs * per || (seqs == 1 && n >= per) || (t.dim() > 0 && t.size(0) > seqs && n == t.size(0) * per);
    }
    // .. and these leading dimensions, with `inner` elements behind them
    void rows_are(int i, int64_t B, int64_t N, int64_t inner) {
        if (!ok || a[i] == Py_None) return;
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        ok = t.size(0) == B && t.size(1) == N && t.numel() == B * N * inner;
    }
    // .. exactly so many rows, with `inner` elements to each
    void flat_rows_are(int i, int64_t N, int64_t inner) {
        if (!ok || a[i] == Py_None) return;
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        ok = t.size(0) == N && t.numel() == N * inner;
    }
    // .. and exactly these dimensions behind a first one that is at least `layers`
    void layers_are(int i, int64_t layers, std::initializer_list<int64_t> behind) {
        if (!ok || a[i] == Py_None) return;
        const at::IntArrayRef z = THPVariable_Unpack(a[i]).sizes();
        ok = z.size() == behind.size() + 1 && z[0] >= layers && std::equal(behind.begin(), behind.end(), z.begin() + 1);
    }
    int32_t size(int i, int64_t d) {   // of a tensor that passed its check, else 0
        if (!ok || a[i] == Py_None) return 0;
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (d >= t.dim() || t.size(d) > INT32_MAX) { ok = false; return 0; }
        return (int32_t)t.size(d);
    }
    bool number(int i, int32_t& out) {
        const int64_t v = PyLong_AsLongLong(a[i]);
        if ((v == -1 && PyErr_Occurred()) || v < INT32_MIN || v > INT32_MAX) { PyErr_Clear(); return ok = false; }
        out = (int32_t)v;
        return true;
    }
};

bool known_type(const ygg_shape& s) { return (s.kv_dtype >= YGG_F32 && s.kv_dtype <= YGG_FP8_BLOCK) || s.kv_dtype == YGG_FP4_BLOCK; }

at::ScalarType kv_type(const ygg_shape& s) {
    return s.kv_dtype == YGG_F32 ? at::kFloat : s.kv_dtype == YGG_FP8_E4M3 ? at::kByte : at::kBFloat16;
}

template <typename F>
PyObject* finish(bool ok, F&& call) {
    if (!ok) return PyLong_FromLong(kCheckFailed);
    void* stream = c10::hip::getCurrentHIPStream().stream();
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS   // a launch waits when the queue is full
    rc = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd positional arguments, got %zd", want, n);
    return false;
}

// (shape, q, k_cache, v_cache, seq_lens, k_tree, v_tree, parent_idx, out, lse, workspace, main_kernel_only)
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 12)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s) && known_type(s);
    const at::ScalarType dt = kv_type(s);
    void *q = t.ptr(1, dt), *kc = t.ptr(2, dt), *vc = t.ptr(3, dt), *kt = t.ptr(5, dt), *vt = t.ptr(6, dt), *out = t.ptr(8, dt);
    int32_t *lens = t.ints(4), *parent = t.ints(7);
    float* lse = t.floats(9);
    size_t wn;
    void* ws = t.scratch(10, wn);
    const bool main_only = a[11] == Py_True;
    return finish(t.ok, [&](void* st) {
        return (main_only ? ygg_debug_tree_attention_main : ygg_tree_attention)(&s, q, kc, vc, lens, kt, vt, parent, out, lse, ws, wn, st);
    });
}

// (shape, q, k_cache, v_cache, seq_lens, k_tree, v_tree, k_scale, v_scale, parent_idx, out, lse, workspace)
PyObject* tree_attention_fp8kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 13)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    void *q = t.ptr(1, at::kBFloat16), *kc = t.ptr(2, at::kByte), *vc = t.ptr(3, at::kByte), *kt = t.ptr(5, at::kByte),
         *vt = t.ptr(6, at::kByte), *out = t.ptr(10, at::kBFloat16);
    int32_t *lens = t.ints(4), *parent = t.ints(9);
    float *ks = t.floats(7), *vs = t.floats(8), *lse = t.floats(11);
    size_t wn;
    void* ws = t.scratch(12, wn);
    return finish(t.ok, [&](void* st) {
        return ygg_tree_attention_fp8kv(&s, q, kc, vc, lens, kt, vt, ks, vs, parent, out, lse, ws, wn, st);
    });
}

// (shape, d, draft_logits, parent_idx, token_ids, cum_logprob, workspace)
PyObject* equal_growth_expand(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int32_t d = 0;
    t.number(1, d);
    float *x = t.floats(2), *cum = t.floats(5);
    int32_t *parent = t.ints(3), *token = t.ints(4);
    size_t wn;
    void* ws = t.scratch(6, wn);
    return finish(t.ok, [&](void* st) { return ygg_equal_growth_expand(&s, d, x, parent, token, cum, ws, wn, st); });
}

// (shape, d, draft_logits, parent_idx, token_ids, cum_logprob)
PyObject* equal_growth_expand_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 6)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int32_t d = 0;
    t.number(1, d);
    float *x = t.floats(2), *cum = t.floats(5);
    int32_t *parent = t.ints(3), *token = t.ints(4);
    return finish(t.ok, [&](void* st) { return ygg_equal_growth_expand_static(&s, d, x, parent, token, cum, st); });
}

// (shape, t, draft_logits, parent_idx, token_ids, cum_logprob, pool, workspace)
PyObject* equal_growth_attach(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 8)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int32_t step = 0;
    t.number(1, step);
    float *x = t.floats(2), *cum = t.floats(5);
    int32_t *parent = t.ints(3), *token = t.ints(4);
    size_t pn, wn;
    void *pool = t.scratch(6, pn), *ws = t.scratch(7, wn);
    return finish(t.ok, [&](void* st) { return ygg_equal_growth_attach(&s, step, x, parent, token, cum, pool, pn, ws, wn, st); });
}

// (shape, w_verify, parent_idx, token_ids, cum_logprob, kept_nodes, new_parent, new_token, expected_len, best_width,
//  t_verifier, t_draft)
PyObject* prune_for_verification(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 12)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int32_t w = 0;
    t.number(1, w);
    int32_t *parent = t.ints(2), *token = t.ints(3), *kept = t.ints(5), *np = t.ints(6), *nt = t.ints(7), *best = t.ints(9);
    float *cum = t.floats(4), *expected = t.floats(8), *tv = t.floats(10);
    const double td = PyFloat_AsDouble(a[11]);
    if (PyErr_Occurred()) { PyErr_Clear(); t.ok = false; }
    return finish(t.ok, [&](void* st) {
        return ygg_prune_for_verification(&s, w, parent, token, cum, tv, (float)td, kept, np, nt, expected, best, st);
    });
}

// (shape, n_layers, parent_idx, token_ids, k_tree, v_tree, k_cache, v_cache, seq_lens, accept_len, accept_path,
//  bonus_token, target_logits, target_tokens, workspace)
PyObject* accept_and_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 15)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s) && known_type(s);
    const at::ScalarType dt = kv_type(s);
    int32_t layers = 0;
    t.number(1, layers);
    int32_t *parent = t.ints(2), *token = t.ints(3), *lens = t.ints(8), *alen = t.ints(9), *path = t.ints(10), *bonus = t.ints(11),
            *tokens = t.ints(13);
    void *kt = t.ptr(4, dt), *vt = t.ptr(5, dt), *kc = t.ptr(6, dt), *vc = t.ptr(7, dt);
    float* logits = t.floats(12);
    size_t wn;
    void* ws = t.scratch(14, wn);
    return finish(t.ok, [&](void* st) {
        return ygg_accept_and_compact(&s, layers, logits, tokens, parent, token, kt, vt, kc, vc, lens, alen, path, bonus, ws, wn, st);
    });
}

// A tensor of a block cache: `per` elements to a sequence in `rank` dimensions, that of the sequences the first, perhaps with a layer
// dimension before them.  The kernels step by the shape's batch and capacity, so further layers and, behind a single layer, further
// sequences may follow; a call for one layer takes no tensor of several, which would have to be its first.
bool cache_part(const at::Tensor& t, int64_t rank, int64_t layers, int64_t batch, int64_t per, bool alone) {
    if (t.numel() == layers * batch * per) return true;
    const bool layered = t.dim() == rank + 1;
    if (!layered && t.dim() != rank) return false;
    const int64_t L = layered ? t.size(0) : 1, B = t.size(layered ? 1 : 0);
    return t.numel() == L * B * per && (alone ? L == 1 : L >= layers) && (L == 1 ? B >= batch : B == batch);
}

// The six tensors of a block cache of so many layers (alone: and no more), from argument i on
template <typename Cache>
Cache block_cache(Args& t, int i, const ygg_shape& s, int64_t layers, bool alone) {
    constexpr bool FOUR = std::is_same<Cache, ygg_block4_cache>::value;
    Cache c{};
    c.k_codes = t.ptr(i, at::kByte); c.v_codes = t.ptr(i + 1, at::kByte);
    using Scale = decltype(c.k_scale);
    c.k_scale = static_cast<Scale>(t.ptr(i + 2, FOUR ? at::kByte : at::kFloat)); c.v_scale = static_cast<Scale>(t.ptr(i + 3, FOUR ? at::kByte : at::kFloat));
    c.k_tail = t.ptr(i + 4, at::kBFloat16); c.v_tail = t.ptr(i + 5, at::kBFloat16);
    const int64_t nblk = (s.kv_capacity + YGG_KV_BLOCK - 1) / YGG_KV_BLOCK, Hkv = s.n_kv_heads, Dh = s.head_dim;
    const int64_t per[3] = {Hkv * nblk * YGG_KV_BLOCK * Dh / (FOUR ? 2 : 1), Hkv * nblk * (FOUR ? 2 * Dh : 1), Hkv * 2 * YGG_KV_BLOCK * Dh};
    const int64_t rank[3] = {4, FOUR ? 4 : 3, 4};
    for (int k = 0; k < 6; ++k)
        if (t.ok && t.a[i + k] != Py_None)
            t.ok = cache_part(THPVariable_Unpack(t.a[i + k]), rank[k / 2], layers, s.batch, per[k / 2], alone);
    return c;
}

template <typename Cache, typename Call>
PyObject* tree_attention_block(PyObject* const* a, Py_ssize_t n, Call call) {
    if (!arity(n, 15)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    const Cache c = block_cache<Cache>(t, 2, s, 1, true);
    void *q = t.ptr(1, at::kBFloat16), *kt = t.ptr(9, at::kBFloat16), *vt = t.ptr(10, at::kBFloat16), *out = t.ptr(12, at::kBFloat16);
    int32_t *lens = t.ints(8), *parent = t.ints(11);
    float* lse = t.floats(13);
    size_t wn;
    void* ws = t.scratch(14, wn);
    const int64_t B = s.batch, N = s.n_nodes;
    for (int i : {1, 12}) t.holds(i, B, N * s.n_q_heads * s.head_dim);
    for (int i : {9, 10}) t.holds(i, B, N * s.n_kv_heads * s.head_dim);
    t.holds(8, B, 1); t.holds(11, B, N); t.holds(13, B, N * s.n_q_heads);
    return finish(t.ok, [&](void* st) { return call(&s, q, &c, lens, kt, vt, parent, out, lse, ws, wn, st); });
}

// (shape, q, k_codes, v_codes, k_scale, v_scale, k_tail, v_tail, seq_lens, k_tree, v_tree, parent_idx, out, lse, workspace)
PyObject* tree_attention_block8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return tree_attention_block<ygg_block8_cache>(a, n, ygg_tree_attention_block8);
}
PyObject* tree_attention_block4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return tree_attention_block<ygg_block4_cache>(a, n, ygg_tree_attention_block4);
}

template <typename Cache, typename Call>
PyObject* block_append(PyObject* const* a, Py_ssize_t n, Call call) {
    if (!arity(n, 13)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int32_t layers = 0;
    t.number(1, layers);
    void *k = t.ptr(2, at::kBFloat16), *v = t.ptr(3, at::kBFloat16);
    int32_t *rows = t.ints(4), *n_new = t.ints(5), *lens = t.ints(6);
    const Cache c = block_cache<Cache>(t, 7, s, layers, false);
    const int32_t n_rows = t.size(2, 2), most = rows ? t.size(4, 1) : n_rows;
    for (int i : {2, 3}) t.layers_are(i, layers, {s.batch, n_rows, s.n_kv_heads, s.head_dim});
    t.holds(4, s.batch, most); t.holds(5, s.batch, 1); t.holds(6, s.batch, 1);
    return finish(t.ok, [&](void* st) { return call(&s, layers, k, v, n_rows, rows, most, n_new, lens, &c, st); });
}

// (shape, n_layers, k_new, v_new, rows, n_new, seq_lens, k_codes, v_codes, k_scale, v_scale, k_tail, v_tail)
PyObject* block8_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return block_append<ygg_block8_cache>(a, n, ygg_block8_append); }
PyObject* block4_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return block_append<ygg_block4_cache>(a, n, ygg_block4_append); }

// (shape, q, k, q_out, k_out, frequencies, seq_lens, parent_idx, positions, interleaved, scale)
PyObject* tree_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 11)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    const at::ScalarType dt = s.kv_dtype == YGG_F32 ? at::kFloat : at::kBFloat16;
    int64_t qs, ks;
    void *q = t.rows(1, dt, qs), *k = t.rows(2, dt, ks), *qo = t.ptr(3, dt), *ko = t.ptr(4, dt);
    const double* f = t.typed<double>(5, at::kDouble);
    const int32_t pairs = t.size(5, 0);
    int32_t *lens = t.ints(6), *parent = t.ints(7), *positions = t.ints(8);
    const int64_t B = s.batch, N = s.n_nodes, q_row = (int64_t)s.n_q_heads * s.head_dim, k_row = (int64_t)s.n_kv_heads * s.head_dim;
    t.rows_are(1, B, N, q_row); t.rows_are(2, B, N, k_row);
    t.holds(3, B, N * q_row); t.holds(4, B, N * k_row); t.holds(8, B, N);
    if (!positions) { t.holds(6, B, 1); t.holds(7, B, N); }   // (else they are not read)
    const bool interleaved = a[9] == Py_True;
    const double scale = PyFloat_AsDouble(a[10]);
    if (PyErr_Occurred()) { PyErr_Clear(); t.ok = false; }
    return finish(t.ok && pairs <= 1024, [&](void* st) {
        return ygg_tree_rotary(&s, q, qs, k, ks, qo, ko, f, 2 * pairs, interleaved, (float)scale, lens, parent, positions, st);
    });
}

// (shape, q, k, q_out, k_out, q_weight, k_weight, frequencies, seq_lens, parent_idx, positions, interleaved, scale, eps)
PyObject* tree_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 14)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    const at::ScalarType dt = s.kv_dtype == YGG_F32 ? at::kFloat : at::kBFloat16;
    int64_t qs, ks;
    void *q = t.rows(1, dt, qs), *k = t.rows(2, dt, ks), *qo = t.ptr(3, dt), *ko = t.ptr(4, dt);
    float *qw = t.floats(5), *kw = t.floats(6);
    const double* f = t.typed<double>(7, at::kDouble);
    const int32_t pairs = t.size(7, 0);
    int32_t *lens = t.ints(8), *parent = t.ints(9), *positions = t.ints(10);
    const int64_t B = s.batch, N = s.n_nodes, Dh = s.head_dim, q_row = s.n_q_heads * Dh, k_row = s.n_kv_heads * Dh;
    t.rows_are(1, B, N, q_row); t.rows_are(2, B, N, k_row);
    t.holds(3, B, N * q_row); t.holds(4, B, N * k_row); t.holds(10, B, N);
    // weights of every head's own have two dimensions, in q's and k's alike
    auto dims = [&](int i) -> int64_t { return t.ok && a[i] != Py_None ? THPVariable_Unpack(a[i]).dim() : 0; };
    const bool per_head = dims(5) == 2 || dims(6) == 2;
    for (int i : {5, 6})
        if (t.ok && a[i] != Py_None) {
            const at::Tensor& w = THPVariable_Unpack(a[i]);
            t.ok = w.dim() == (per_head ? 2 : 1) && w.size(-1) == Dh && (!per_head || w.size(0) == (i == 5 ? s.n_q_heads : s.n_kv_heads));
        }
    if (!positions) { t.holds(8, B, 1); t.holds(9, B, N); }   // (else they are not read)
    const bool interleaved = a[11] == Py_True;
    const double scale = PyFloat_AsDouble(a[12]);
    const double eps = PyErr_Occurred() ? -1.0 : PyFloat_AsDouble(a[13]);
    if (PyErr_Occurred()) { PyErr_Clear(); t.ok = false; }
    return finish(t.ok && pairs <= 1024, [&](void* st) {
        return ygg_tree_norm_rotary(&s, q, qs, k, ks, qo, ko, qw, kw, per_head, (float)eps, f, 2 * pairs, interleaved, (float)scale, lens, parent,
                                    positions, st);
    });
}

// (shape, q, k, v, q_first, q_len, k_first, k_len, out, lse, workspace)
PyObject* prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 11)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    const at::ScalarType dt = s.kv_dtype == YGG_F32 ? at::kFloat : at::kBFloat16;
    int64_t qs, ks, vs;
    void *q = t.flat_rows(1, dt, qs), *k = t.flat_rows(2, dt, ks), *v = t.flat_rows(3, dt, vs), *out = t.ptr(8, dt);
    int32_t *qf = t.ints(4), *ql = t.ints(5), *kf = t.ints(6), *kl = t.ints(7);
    float* lse = t.floats(9);
    size_t wn;
    void* ws = t.scratch(10, wn);
    const int64_t N = s.n_nodes, q_row = (int64_t)s.n_q_heads * s.head_dim, k_row = (int64_t)s.n_kv_heads * s.head_dim;
    t.flat_rows_are(1, N, q_row);
    for (int i : {2, 3}) t.flat_rows_are(i, s.kv_capacity, k_row);
    t.holds(8, 1, N * q_row); t.holds(9, 1, N * s.n_q_heads);
    for (int i : {4, 5, 6, 7}) t.holds(i, s.batch, 1);
    return finish(t.ok, [&](void* st) { return ygg_prompt_attention(&s, q, qs, k, ks, v, vs, qf, ql, kf, kl, out, lse, ws, wn, st); });
}

// (shape, tokens, n_new, counts, rows, first, prompt)
PyObject* count_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int32_t *tokens = t.ints(1), *n_new = t.ints(2), *counts = t.ints(3), *rows = t.ints(4);
    int32_t first = 0;
    t.number(5, first);
    const int32_t n_tokens = t.size(1, 1), most = rows ? t.size(4, 1) : n_tokens;
    t.holds(1, s.batch, n_tokens); t.holds(2, s.batch, 1); t.holds(3, s.batch, s.vocab); t.holds(4, s.batch, most);
    const bool prompt = a[6] == Py_True;
    return finish(t.ok, [&](void* st) { return ygg_count_tokens(&s, tokens, n_tokens, rows, first, most, n_new, prompt, counts, st); });
}

// (shape, logits, parent_idx, token_ids, out, best, counts, repetition, presence, frequency, bias, masks, mask_index, workspace)
PyObject* constrain_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 14)) return nullptr;
    ygg_shape s{};
    Args t{a};
    t.ok = read_shape(a[0], s);
    int64_t stride;
    void* x = t.rows(1, at::kFloat, stride, true);
    int32_t dt = -1;
    if (t.ok && x) {
        const at::ScalarType type = THPVariable_Unpack(a[1]).scalar_type();
        dt = type == at::kFloat ? YGG_F32 : type == at::kBFloat16 ? YGG_BF16 : -1;
        t.ok = dt >= 0;
    }
    int32_t *parent = t.ints(2), *token = t.ints(3), *best = t.ints(5);
    float* out = t.floats(4);
    ygg_logit_rules r{};
    r.counts = t.ints(6);
    r.repetition = t.floats(7); r.presence = t.floats(8); r.frequency = t.floats(9); r.bias = t.floats(10);
    r.bias_shared = r.bias && t.ok && THPVariable_Unpack(a[10]).dim() == 1;
    r.masks = reinterpret_cast<const uint32_t*>(t.ints(11));
    r.n_masks = t.size(11, 0);
    r.mask_index = t.ints(12);
    const int64_t B = s.batch, N = s.n_nodes, V = s.vocab;
    t.rows_are(1, B, N, V);
    for (int i : {2, 3, 5, 12}) t.holds(i, B, N);
    for (int i : {7, 8, 9}) t.holds(i, B, 1);
    t.holds(4, B, N * V); t.holds(6, B, V); t.holds(10, r.bias_shared ? 1 : B, V); t.holds(11, r.n_masks, (V + 31) / 32);
    size_t wn;
    void* ws = t.scratch(13, wn);
    return finish(t.ok, [&](void* st) { return ygg_constrain_logits(&s, x, dt, stride, parent, token, &r, out, best, ws, wn, st); });
}

// torch reports its errors (no device, a tensor without storage) as C++ exceptions
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    try {
        return F(self, a, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define YGG_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    YGG_CALL(tree_attention), YGG_CALL(tree_attention_fp8kv), YGG_CALL(equal_growth_expand), YGG_CALL(equal_growth_expand_static),
    YGG_CALL(equal_growth_attach), YGG_CALL(prune_for_verification), YGG_CALL(accept_and_compact),
    YGG_CALL(tree_attention_block8), YGG_CALL(block8_append), YGG_CALL(tree_rotary), YGG_CALL(count_tokens),
    YGG_CALL(constrain_logits), YGG_CALL(tree_norm_rotary), YGG_CALL(prompt_attention), YGG_CALL(block4_append),
    YGG_CALL(tree_attention_block4), {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", "native argument marshalling of the launching calls", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
    for (int i = 0; i < 12; ++i)
        if (!(g_field[i] = PyUnicode_InternFromString(kField[i]))) return nullptr;
    return PyModule_Create(&kModule);
}
