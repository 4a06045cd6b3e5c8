// Marshalling of the calls of a serving loop: the arguments of a schedule or apply call, as torch tensors, to the C ABI.
//
// A ctypes call of 21 arguments, with every property of ten tensors asked for from Python, takes 4 to 7 us beside the 3 us of
// the launch itself; a launch of 6 us waits for it.  Here the same takes below 1 us, also with the slot manager's pools (binding.PoolRef) and with
// numbers of any type.  Anything else -- a tensor subclass, another table, a check that fails, an exception of torch -- answers None, and the
// caller goes through binding.py's own path, which makes the same checks and raises what they raise.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/preft.h"

namespace {

decltype(&preft_schedule) g_schedule;
decltype(&preft_lora_apply) g_lora;
decltype(&preft_lora_apply_packed) g_packed;
decltype(&preft_direft_apply) g_direft;
decltype(&preft_loreft_apply) g_loreft;
decltype(&preft_direft_apply_layers) g_layers;
decltype(&preft_kv_plan) g_plan;
decltype(&preft_kv_store) g_store;
decltype(&preft_prompt_attention) g_prompt;
decltype(&preft_cached_attention) g_cached, g_cached_mx;
decltype(&preft_qk_rotate) g_rotate;
decltype(&preft_kv_append) g_append, g_append4;
decltype(&preft_kv_fetch_mx) g_fetch;

const at::Tensor *tensor(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

struct Matrix { void *p; int64_t ld; int32_t rows, cols; at::ScalarType type; };

bool as_matrix(PyObject *o, Matrix &m)
{
    const at::Tensor *t = tensor(o);
    if (!t || t->dim() != 2 || !t->is_cuda() || t->stride(1) != 1) return false;
    if (t->size(0) > INT32_MAX || t->size(1) > INT32_MAX) return false;
    m = {t->data_ptr(), t->stride(0), (int32_t)t->size(0), (int32_t)t->size(1), t->scalar_type()};
    return m.type == at::kBFloat16 || m.type == at::kFloat;
}

// a contiguous device table of n entries
template <typename T>
bool as_table(PyObject *o, int64_t n, T *&p)
{
    const at::Tensor *t = tensor(o);
    if (!t || t->scalar_type() != (sizeof(T) == 4 ? at::kInt : at::kLong) || t->numel() != n || !t->is_cuda() || !t->is_contiguous()) return false;
    p = static_cast<T *>(t->data_ptr());
    return true;
}

struct Segments { int32_t *start, *adapter, *prefill, S; };

bool as_segments(PyObject *const *o, Segments &s)
{
    const at::Tensor *t = tensor(o[1]);
    if (!t || t->numel() >= INT32_MAX) return false;
    s.S = (int32_t)t->numel();
    return as_table(o[0], (int64_t)s.S + 1, s.start) && as_table(o[1], s.S, s.adapter) && as_table(o[2], s.S, s.prefill);
}

PyObject *g_pool_ref, *g_address, *g_length;                  // binding.PoolRef, and the names of what it holds

bool as_pool_ref(PyObject *o, int64_t &n, const void *const *&p)
{
    if ((PyObject *)Py_TYPE(o) != g_pool_ref) return false;
    PyObject *address = PyObject_GetAttr(o, g_address), *length = address ? PyObject_GetAttr(o, g_length) : nullptr;
    bool ok = length && PyLong_CheckExact(address) && PyLong_CheckExact(length);
    if (ok) {
        void *at = PyLong_AsVoidPtr(address);
        const long long count = PyLong_AsLongLong(length);
        ok = !PyErr_Occurred() && count >= 0 && count <= INT32_MAX && (n < 0 || count == n);
        if (ok) { p = static_cast<const void *const *>(at); n = count; }
    }
    Py_XDECREF(address);
    Py_XDECREF(length);
    return ok;
}

bool as_pool(PyObject *o, int64_t &n, const void *const *&p)      // n < 0: any length
{
    if (as_pool_ref(o, n, p)) return true;
    const at::Tensor *t = tensor(o);
    if (!t || t->scalar_type() != at::kLong || (n >= 0 && t->numel() != n) || t->numel() > INT32_MAX) return false;
    n = t->numel();
    p = static_cast<const void *const *>(t->data_ptr());
    return true;
}

bool as_int(PyObject *o, int32_t &v)
{
    int overflow = 0;
    long long x;
    if (PyLong_CheckExact(o)) {
        x = PyLong_AsLongLongAndOverflow(o, &overflow);
    } else {                                                  // whole numbers of other types: NumPy's, truth values
        PyObject *i = PyIndex_Check(o) ? PyNumber_Index(o) : nullptr;
        if (!i) return false;
        x = PyLong_AsLongLongAndOverflow(i, &overflow);
        Py_DECREF(i);
    }
    if (overflow || x < INT32_MIN || x > INT32_MAX) return false;
    v = (int32_t)x;
    return true;
}

// what every apply call ends with: rank, scale, mode, workspace, stream, further mode bits
struct Rest { int32_t rank, mode, extra; float scale; void *workspace, *stream; size_t bytes; };

bool as_workspace(PyObject *o, void *&p, size_t &bytes)
{
    const at::Tensor *t = tensor(o);
    if (!t) return false;
    p = t->data_ptr();
    bytes = (size_t)t->numel() * t->element_size();
    return true;
}

bool as_stream(PyObject *o, void *&p)
{
    if (!PyLong_CheckExact(o)) return false;
    p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

bool as_rest(PyObject *const *o, Rest &r)
{
    if (!as_int(o[0], r.rank) || !as_int(o[2], r.mode) || !as_int(o[5], r.extra)) return false;
    const double scale = PyFloat_AsDouble(o[1]);              // whole numbers and NumPy's too
    if (scale == -1.0 && PyErr_Occurred()) return false;
    r.scale = (float)scale;
    r.mode |= r.extra;
    return as_workspace(o[3], r.workspace, r.bytes) && as_stream(o[4], r.stream);
}

int dtype_of(at::ScalarType t) { return t == at::kBFloat16 ? PREFT_BF16 : PREFT_F32; }

template <typename F>
PyObject *answer(F call)
{
    try {
        int rc = 0;
        if (call(rc)) return PyLong_FromLong(rc);
    } catch (...) {                                           // the caller's own path says what is wrong
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

template <typename F>
int without_gil(F launch)
{
    PyThreadState *state = PyEval_SaveThread();
    const int rc = launch();
    PyEval_RestoreThread(state);
    return rc;
}

// (workspace, seg_start, seg_adapter, seg_prefill_len, T, N, mode, stream)
PyObject *schedule(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Segments s;
        void *ws, *stream;
        size_t bytes;
        int32_t T, N, mode;
        if (n != 8 || !g_schedule || !as_workspace(o[0], ws, bytes) || !as_segments(o + 1, s) || !as_int(o[4], T) || !as_int(o[5], N) ||
            !as_int(o[6], mode) || !as_stream(o[7], stream)) return false;
        rc = without_gil([&] { return g_schedule(ws, bytes, s.start, s.adapter, s.prefill, s.S, T, N, mode, stream); });
        return true;
    });
}

// (y, x, seg_start, seg_adapter, seg_prefill_len, A_pool, B_pool, rest ...)
PyObject *lora(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Matrix y, x;
        Segments s;
        Rest r;
        int64_t N = -1;
        const void *const *A, *const *B;
        if (n != 13 || !g_lora || !as_matrix(o[0], y) || !as_matrix(o[1], x) || y.rows != x.rows || y.type != x.type || !as_segments(o + 2, s) ||
            !as_pool(o[5], N, A) || !as_pool(o[6], N, B) || !as_rest(o + 7, r)) return false;
        rc = without_gil([&] {
            return g_lora(y.p, y.ld, x.p, x.ld, y.rows, x.cols, y.cols, s.start, s.adapter, s.prefill, s.S, A, B, (int32_t)N, r.rank, r.scale,
                          dtype_of(y.type), r.mode, r.workspace, r.bytes, r.stream);
        });
        return true;
    });
}

// (ys, x, seg_start, seg_adapter, seg_prefill_len, A_pools, B_pools, rest ...); ys and the pools lists or tuples
PyObject *lora_packed(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        auto sequence = [](PyObject *v) { return PyList_CheckExact(v) || PyTuple_CheckExact(v); };
        if (n != 13 || !g_packed || !sequence(o[0]) || !sequence(o[5]) || !sequence(o[6])) return false;
        const Py_ssize_t k = PySequence_Fast_GET_SIZE(o[0]);
        if (k < 1 || k > PREFT_MAX_PACKED || PySequence_Fast_GET_SIZE(o[5]) != k || PySequence_Fast_GET_SIZE(o[6]) != k) return false;
        Matrix x, y;
        Segments s;
        Rest r;
        int64_t N = -1, ld[PREFT_MAX_PACKED];
        void *yp[PREFT_MAX_PACKED];
        int32_t d_out[PREFT_MAX_PACKED];
        const void *const *A[PREFT_MAX_PACKED], *const *B[PREFT_MAX_PACKED];
        if (!as_matrix(o[1], x) || !as_segments(o + 2, s) || !as_rest(o + 7, r)) return false;
        for (Py_ssize_t i = 0; i < k; ++i) {
            if (!as_matrix(PySequence_Fast_GET_ITEM(o[0], i), y) || y.rows != x.rows || y.type != x.type ||
                !as_pool(PySequence_Fast_GET_ITEM(o[5], i), N, A[i]) || !as_pool(PySequence_Fast_GET_ITEM(o[6], i), N, B[i])) return false;
            yp[i] = y.p; ld[i] = y.ld; d_out[i] = y.cols;
        }
        rc = without_gil([&] {
            return g_packed((int32_t)k, yp, ld, d_out, x.p, x.ld, x.rows, x.cols, s.start, s.adapter, s.prefill, s.S, A, B, (int32_t)N, r.rank,
                            r.scale, dtype_of(x.type), r.mode, r.workspace, r.bytes, r.stream);
        });
        return true;
    });
}

// (loreft, h, seg_start, seg_adapter, seg_prefill_len, W1_pool, W2t_pool, b_pool or None, rest ...)
PyObject *reft(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Matrix h;
        Segments s;
        Rest r;
        int64_t N = -1;
        const void *const *W1, *const *W2t, *const *b = nullptr;
        if (n != 14 || !g_direft || !g_loreft || !as_matrix(o[1], h) || !as_segments(o + 2, s) || !as_pool(o[5], N, W1) || !as_pool(o[6], N, W2t) ||
            (o[7] != Py_None && !as_pool(o[7], N, b)) || !as_rest(o + 8, r)) return false;
        const auto entry = o[0] == Py_True ? g_loreft : g_direft;
        rc = without_gil([&] {
            return entry(h.p, h.ld, h.rows, h.cols, s.start, s.adapter, s.prefill, s.S, W1, W2t, b, (int32_t)N, r.rank, r.scale, dtype_of(h.type),
                         r.mode, r.workspace, r.bytes, r.stream);
        });
        return true;
    });
}

// (hs, h_layers, seg_start, seg_adapter, seg_prefill_len, W1_pools, W2t_pools, b_pools or None, N, rest ...); hs a list or tuple
PyObject *reft_layers(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        if (n != 15 || !g_layers || !(PyList_CheckExact(o[0]) || PyTuple_CheckExact(o[0]))) return false;
        const Py_ssize_t L = PySequence_Fast_GET_SIZE(o[0]);
        if (L < 1 || L > PREFT_MAX_LAYERS) return false;
        Matrix h, first;
        for (Py_ssize_t i = 0; i < L; ++i) {
            if (!as_matrix(PySequence_Fast_GET_ITEM(o[0], i), h)) return false;
            if (i == 0) first = h;
            if (h.ld != first.ld || h.rows != first.rows || h.cols != first.cols || h.type != first.type) return false;
        }
        Segments s;
        Rest r;
        int32_t N;
        int64_t *table, *W1, *W2t, *b = nullptr;
        if (!as_table(o[1], L, table) || !as_segments(o + 2, s) || !as_table(o[5], L, W1) || !as_table(o[6], L, W2t) ||
            (o[7] != Py_None && !as_table(o[7], L, b)) || !as_int(o[8], N) || !as_rest(o + 9, r)) return false;
        using Pools = const void *const *const *;
        rc = without_gil([&] {
            return g_layers(reinterpret_cast<void *const *>(table), h.ld, (int32_t)L, h.rows, h.cols, s.start, s.adapter, s.prefill, s.S,
                            reinterpret_cast<Pools>(W1), reinterpret_cast<Pools>(W2t), reinterpret_cast<Pools>(b), N, r.rank, r.scale,
                            dtype_of(h.type), r.mode, r.workspace, r.bytes, r.stream);
        });
        return true;
    });
}

struct Pages { int32_t *p, max_pages; int64_t ld; };

// int32 device tensor of S rows, unit column stride
bool as_block_table(PyObject *o, int32_t S, Pages &b)
{
    const at::Tensor *t = tensor(o);
    if (!t || t->dim() != 2 || t->scalar_type() != at::kInt || !t->is_cuda() || t->size(0) != S || t->size(1) > INT32_MAX ||
        (t->size(1) > 1 && t->stride(1) != 1)) return false;
    b = {static_cast<int32_t *>(t->data_ptr()), (int32_t)t->size(1), S > 1 ? t->stride(0) : t->size(1)};
    return true;
}

struct Cache { void *k, *v; int32_t n_pages, heads, page, dim; at::ScalarType type; };

// contiguous device tensors [n_pages, n_kv_heads, page_size, head_dim]
bool as_cache(PyObject *ko, PyObject *vo, Cache &c)
{
    const at::Tensor *k = tensor(ko), *v = tensor(vo);
    if (!k || !v || k->dim() != 4 || !k->is_cuda() || !v->is_cuda() || !k->is_contiguous() || !v->is_contiguous() || k->sizes() != v->sizes() ||
        k->scalar_type() != v->scalar_type()) return false;
    for (int i = 0; i < 4; ++i)
        if (k->size(i) > INT32_MAX) return false;
    c = {k->data_ptr(), v->data_ptr(), (int32_t)k->size(0), (int32_t)k->size(1), (int32_t)k->size(2), (int32_t)k->size(3), k->scalar_type()};
    return c.type == at::kBFloat16 || c.type == at::kFloat;
}

// entries of a one-dimensional table, or -1
int64_t entries(PyObject *o)
{
    const at::Tensor *t = tensor(o);
    return t && t->numel() < INT32_MAX ? t->numel() : -1;
}

// (slot_map, positions, kv_len, block_table, counts, seg_start, ctx_len, free_pages, page_size, stream)
PyObject *kv_plan(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        if (n != 10 || !g_plan) return false;
        const int64_t S = entries(o[6]), T = entries(o[0]), n_free = entries(o[7]);
        int64_t *slots;
        int32_t *positions, *kv_len, *counts, *start, *ctx, *free_pages, page;
        Pages b;
        void *stream;
        if (S < 0 || T < 0 || n_free < 0 || !as_table(o[0], T, slots) || !as_table(o[1], T, positions) || !as_table(o[2], S, kv_len) ||
            !as_block_table(o[3], (int32_t)S, b) || !as_table(o[4], 2, counts) || !as_table(o[5], S + 1, start) || !as_table(o[6], S, ctx) ||
            !as_table(o[7], n_free, free_pages) || !as_int(o[8], page) || !as_stream(o[9], stream)) return false;
        rc = without_gil([&] {
            return g_plan(slots, positions, kv_len, b.p, b.ld, b.max_pages, counts, start, ctx, (int32_t)S, (int32_t)T, free_pages, (int32_t)n_free, page,
                          stream);
        });
        return true;
    });
}

// (k_cache, v_cache, k, v, slot_map, stream)
PyObject *kv_store(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Cache c;
        Matrix k, v;
        int64_t *slots;
        void *stream;
        if (n != 6 || !g_store || !as_cache(o[0], o[1], c) || !as_matrix(o[2], k) || !as_matrix(o[3], v) || k.rows != v.rows || k.cols != v.cols ||
            k.cols != (int64_t)c.heads * c.dim || k.type != c.type || v.type != c.type || !as_table(o[4], k.rows, slots) || !as_stream(o[5], stream))
            return false;
        rc = without_gil([&] { return g_store(c.k, c.v, c.n_pages, c.page, k.p, k.ld, v.p, v.ld, k.rows, c.heads, c.dim, slots, dtype_of(c.type), stream); });
        return true;
    });
}

// scale, mode, workspace, stream
struct Last { float scale; int32_t mode; void *workspace, *stream; size_t bytes; };

bool as_last(PyObject *const *o, Last &l)
{
    const double scale = PyFloat_AsDouble(o[0]);
    if (scale == -1.0 && PyErr_Occurred()) return false;
    l.scale = (float)scale;
    const at::Tensor *ws = tensor(o[2]);
    if (!ws || !ws->is_cuda() || !ws->is_contiguous()) return false;
    return as_int(o[1], l.mode) && as_workspace(o[2], l.workspace, l.bytes) && as_stream(o[3], l.stream);
}

// (out, q, k, v, seg_start, seg_prefill_len, n_heads, n_kv_heads, scale, mode, workspace, stream)
PyObject *prompt_attention(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Matrix out, q, k, v;
        int32_t heads, kv_heads, *start, *prefill;
        Last l;
        if (n != 12 || !g_prompt || !as_matrix(o[0], out) || !as_matrix(o[1], q) || !as_matrix(o[2], k) || !as_matrix(o[3], v)) return false;
        const int64_t S = entries(o[5]);
        if (S < 0 || !as_table(o[4], S + 1, start) || !as_table(o[5], S, prefill) || !as_int(o[6], heads) || !as_int(o[7], kv_heads) || !as_last(o + 8, l))
            return false;
        if (heads < 1 || kv_heads < 1 || out.cols % heads != 0 || q.cols != out.cols || k.cols != (int64_t)kv_heads * (out.cols / heads) ||
            v.cols != k.cols || q.rows != out.rows || k.rows != out.rows || v.rows != out.rows || q.type != out.type || k.type != out.type ||
            v.type != out.type) return false;
        rc = without_gil([&] {
            return g_prompt(out.p, out.ld, q.p, q.ld, k.p, k.ld, v.p, v.ld, out.rows, heads, kv_heads, out.cols / heads, start, prefill, (int32_t)S,
                            l.scale, dtype_of(out.type), l.mode, l.workspace, l.bytes, l.stream);
        });
        return true;
    });
}

// contiguous byte tensors [n_pages, n_kv_heads, page_size, head_dim / 2 + head_dim / 32]
bool as_mx4_cache(PyObject *ko, PyObject *vo, Cache &c)
{
    const at::Tensor *k = tensor(ko), *v = tensor(vo);
    if (!k || !v || k->dim() != 4 || !k->is_cuda() || !v->is_cuda() || !k->is_contiguous() || !v->is_contiguous() || k->sizes() != v->sizes() ||
        k->scalar_type() != at::kByte || v->scalar_type() != at::kByte || k->size(3) * 32 % 17 != 0) return false;
    for (int i = 0; i < 4; ++i)
        if (k->size(i) > INT32_MAX / 32) return false;
    c = {k->data_ptr(), v->data_ptr(), (int32_t)k->size(0), (int32_t)k->size(1), (int32_t)k->size(2), (int32_t)(k->size(3) * 32 / 17), at::kByte};
    return true;
}

// (out, q, seg_start, seg_prefill_len or None, kv_len, k_cache, v_cache, block_table, group_start or None, group_prefix_len or None, n_heads, scale,
//  mode, workspace, stream)
template <bool MX>
PyObject *cached_attention(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Matrix out, q;
        Cache c;
        Pages b;
        int32_t heads, *start, *prefill = nullptr, *kv_len, *groups = nullptr, *prefix = nullptr;
        Last l;
        const auto entry = MX ? g_cached_mx : g_cached;
        if (n != 15 || !entry || !as_matrix(o[0], out) || !as_matrix(o[1], q)) return false;
        const int64_t S = entries(o[4]);
        if (S < 0 || !as_table(o[2], S + 1, start) || (o[3] != Py_None && !as_table(o[3], S, prefill)) || !as_table(o[4], S, kv_len) ||
            !(MX ? as_mx4_cache(o[5], o[6], c) : as_cache(o[5], o[6], c)) || !as_block_table(o[7], (int32_t)S, b) || !as_int(o[10], heads) || !as_last(o + 11, l)) return false;
        if ((o[8] == Py_None) != (o[9] == Py_None)) return false;
        const int64_t n_groups = o[9] == Py_None ? 0 : entries(o[9]);
        if (n_groups < 0 || (n_groups > 0 && (!as_table(o[8], n_groups + 1, groups) || !as_table(o[9], n_groups, prefix)))) return false;
        if (heads < 1 || out.cols != (int64_t)heads * c.dim || q.cols != out.cols || q.rows != out.rows || q.type != out.type || (!MX && c.type != out.type))
            return false;
        rc = without_gil([&] {
            return entry(out.p, out.ld, q.p, q.ld, out.rows, heads, c.heads, c.dim, start, prefill, kv_len, (int32_t)S, c.k, c.v, c.n_pages, c.page,
                            b.p, b.ld, b.max_pages, groups, prefix, (int32_t)n_groups, l.scale, dtype_of(out.type), l.mode, l.workspace, l.bytes, l.stream);
        });
        return true;
    });
}

// heads and what they become; None and None: none
struct HeadRows { Matrix out, in; };

bool as_head_rows(PyObject *out, PyObject *in, int32_t heads, int32_t dim, int32_t T, at::ScalarType type, bool optional, HeadRows &r)
{
    r = {};
    if (in == Py_None) return out == Py_None;
    if (!as_matrix(in, r.in) || r.in.cols != (int64_t)heads * dim || r.in.rows != T || r.in.type != type) return false;
    if (out == Py_None && optional) return true;
    return as_matrix(out, r.out) && r.out.cols == r.in.cols && r.out.rows == T && r.out.type == type;
}

// (positions or None, rotation or None) and (q_weight or None, k_weight or None, eps, pairs, stream)
struct Turned { int32_t *positions; const float *rotation; int32_t n, rot, pairs; const void *weights[2]; float eps; void *stream; };

bool as_turned(PyObject *const *o, PyObject *const *w, int32_t T, int32_t dim, at::ScalarType type, Turned &t)
{
    t = {};
    if (o[0] != Py_None && !as_table(o[0], T, t.positions)) return false;
    if (o[1] != Py_None) {
        const at::Tensor *r = tensor(o[1]);
        if (!r || r->dim() != 2 || r->scalar_type() != at::kFloat || !r->is_cuda() || !r->is_contiguous() || r->size(0) > INT32_MAX || r->size(1) > INT32_MAX ||
            o[0] == Py_None) return false;
        t.rotation = static_cast<const float *>(r->data_ptr());
        t.n = (int32_t)r->size(0);
        t.rot = (int32_t)r->size(1);
    }
    for (int i = 0; i < 2; ++i) {
        if (w[i] == Py_None) continue;
        const at::Tensor *x = tensor(w[i]);
        if (!x || x->scalar_type() != type || x->numel() != dim || !x->is_cuda() || !x->is_contiguous()) return false;
        t.weights[i] = x->data_ptr();
    }
    const double eps = PyFloat_AsDouble(w[2]);
    if (eps == -1.0 && PyErr_Occurred()) return false;
    t.eps = (float)eps;
    return as_int(w[3], t.pairs) && as_stream(w[4], t.stream);
}

// (q_out, q, k_out, k, positions or None, rotation or None, n_heads, n_kv_heads, q_weight or None, k_weight or None, eps, pairs, stream); q or k may be None
PyObject *qk_rotate(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        int32_t heads, kv_heads;
        if (n != 13 || !g_rotate || !as_int(o[6], heads) || !as_int(o[7], kv_heads)) return false;
        const bool has_q = o[1] != Py_None;
        Matrix some;
        if (!as_matrix(has_q ? o[1] : o[3], some)) return false;
        const int32_t of = has_q ? heads : kv_heads;
        if (of < 1 || some.cols % of != 0) return false;
        const int32_t dim = some.cols / of;
        HeadRows q, k;
        Turned t;
        if (!as_head_rows(o[0], o[1], heads, dim, some.rows, some.type, false, q) || !as_head_rows(o[2], o[3], kv_heads, dim, some.rows, some.type, false, k) ||
            !as_turned(o + 4, o + 8, some.rows, dim, some.type, t)) return false;
        if (!has_q) heads = 0;
        if (o[3] == Py_None) kv_heads = 0;
        rc = without_gil([&] {
            return g_rotate(q.out.p, q.out.ld, q.in.p, q.in.ld, k.out.p, k.out.ld, k.in.p, k.in.ld, some.rows, heads, kv_heads, dim, t.weights[0], t.weights[1],
                            t.eps, t.positions, t.rotation, t.n, t.rot, t.pairs, dtype_of(some.type), t.stream);
        });
        return true;
    });
}

// (4-bit pages, k_cache, v_cache, q_out, q, k_out, k, v, slot_map, positions or None, rotation or None, n_heads, q_weight or None, k_weight or None, eps, pairs, stream);
// q_out and q, or k_out, may be None
PyObject *kv_append(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        if (n != 17) return false;
        const bool mx4 = o[0] == Py_True;
        const auto entry = mx4 ? g_append4 : g_append;
        Cache c;
        Matrix v;
        HeadRows q, k;
        Turned t;
        int32_t heads;
        int64_t *slots;
        if (!entry || !(mx4 ? as_mx4_cache(o[1], o[2], c) : as_cache(o[1], o[2], c)) || !as_matrix(o[7], v) || v.cols != (int64_t)c.heads * c.dim ||
            (!mx4 && v.type != c.type) || !as_int(o[11], heads) || o[6] == Py_None || !as_head_rows(o[3], o[4], heads, c.dim, v.rows, v.type, false, q) ||
            !as_head_rows(o[5], o[6], c.heads, c.dim, v.rows, v.type, true, k) || !as_table(o[8], v.rows, slots) ||
            !as_turned(o + 9, o + 12, v.rows, c.dim, v.type, t)) return false;
        if (o[4] == Py_None) heads = 0;
        rc = without_gil([&] {
            return entry(c.k, c.v, c.n_pages, c.page, q.out.p, q.out.ld, q.in.p, q.in.ld, k.out.p, k.out.ld, k.in.p, k.in.ld, v.p, v.ld, v.rows, heads, c.heads,
                         c.dim, slots, t.weights[0], t.weights[1], t.eps, t.positions, t.rotation, t.n, t.rot, t.pairs, dtype_of(v.type), t.stream);
        });
        return true;
    });
}

// (k, v, slot_map, k_cache, v_cache, stream)
PyObject *kv_fetch(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return answer([&](int &rc) {
        Cache c;
        Matrix k, v;
        int64_t *slots;
        void *stream;
        if (n != 6 || !g_fetch || !as_matrix(o[0], k) || !as_matrix(o[1], v) || !as_mx4_cache(o[3], o[4], c) || k.rows != v.rows || k.cols != v.cols ||
            k.cols != (int64_t)c.heads * c.dim || k.type != v.type || !as_table(o[2], k.rows, slots) || !as_stream(o[5], stream)) return false;
        rc = without_gil([&] { return g_fetch(k.p, k.ld, v.p, v.ld, k.rows, c.heads, c.dim, slots, c.k, c.v, c.n_pages, c.page, dtype_of(k.type), stream); });
        return true;
    });
}

// the addresses of preft_qk_rotate, preft_kv_append, preft_kv_append_mx, preft_kv_fetch_mx and preft_cached_attention_mx
PyObject *bind_heads(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    void *p[5];
    if (n != 5) { PyErr_SetString(PyExc_TypeError, "five addresses"); return nullptr; }
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(o[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_rotate = reinterpret_cast<decltype(g_rotate)>(p[0]);
    g_append = reinterpret_cast<decltype(g_append)>(p[1]);
    g_append4 = reinterpret_cast<decltype(g_append4)>(p[2]);
    g_fetch = reinterpret_cast<decltype(g_fetch)>(p[3]);
    g_cached_mx = reinterpret_cast<decltype(g_cached_mx)>(p[4]);
    Py_RETURN_NONE;
}

// the addresses of preft_kv_plan, preft_kv_store, preft_prompt_attention and preft_cached_attention
PyObject *bind_attention(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    void *p[4];
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "four addresses"); return nullptr; }
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(o[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_plan = reinterpret_cast<decltype(g_plan)>(p[0]);
    g_store = reinterpret_cast<decltype(g_store)>(p[1]);
    g_prompt = reinterpret_cast<decltype(g_prompt)>(p[2]);
    g_cached = reinterpret_cast<decltype(g_cached)>(p[3]);
    Py_RETURN_NONE;
}

// binding.PoolRef, and the addresses of the loaded library's entry points in the order below
PyObject *bind(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    void *p[6];
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "a class and six addresses"); return nullptr; }
    PyObject *const pool_ref = *o++;
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(o[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_schedule = reinterpret_cast<decltype(g_schedule)>(p[0]);
    g_lora = reinterpret_cast<decltype(g_lora)>(p[1]);
    g_packed = reinterpret_cast<decltype(g_packed)>(p[2]);
    g_direft = reinterpret_cast<decltype(g_direft)>(p[3]);
    g_loreft = reinterpret_cast<decltype(g_loreft)>(p[4]);
    g_layers = reinterpret_cast<decltype(g_layers)>(p[5]);
    if (!g_address) g_address = PyUnicode_InternFromString("_address");
    if (!g_length) g_length = PyUnicode_InternFromString("_n");
    if (!g_address || !g_length) return nullptr;
    Py_INCREF(pool_ref);
    Py_XDECREF(g_pool_ref);
    g_pool_ref = pool_ref;
    Py_RETURN_NONE;
}

// What it was compiled against (build.py): sizes, strides and addresses are read at that torch's and Python's offsets
PyObject *built_for(PyObject *, PyObject *) { return PyUnicode_FromString(PREFT_BUILT_FOR); }

PyMethodDef methods[] = {
    {"built_for", built_for, METH_NOARGS, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"schedule", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(schedule)), METH_FASTCALL, nullptr},
    {"lora", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(lora)), METH_FASTCALL, nullptr},
    {"lora_packed", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(lora_packed)), METH_FASTCALL, nullptr},
    {"reft", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(reft)), METH_FASTCALL, nullptr},
    {"reft_layers", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(reft_layers)), METH_FASTCALL, nullptr},
    {"kv_plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(kv_plan)), METH_FASTCALL, nullptr},
    {"kv_store", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(kv_store)), METH_FASTCALL, nullptr},
    {"prompt_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(prompt_attention)), METH_FASTCALL, nullptr},
    {"cached_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cached_attention<false>)), METH_FASTCALL, nullptr},
    {"cached_attention_mx", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cached_attention<true>)), METH_FASTCALL, nullptr},
    {"qk_rotate", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(qk_rotate)), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(kv_append)), METH_FASTCALL, nullptr},
    {"kv_fetch", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(kv_fetch)), METH_FASTCALL, nullptr},
    {"bind_heads", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_heads)), METH_FASTCALL, nullptr},
    {"bind_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
