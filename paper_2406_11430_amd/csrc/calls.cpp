// The checks and the argument marshalling of the calls a decode step (also of drafted tokens) and a small compression are made of, for
// the Python binding.  In Python they take 2.5 us a call, with many tensors 7, most of it single reads of tensor attributes, and ctypes
// another 0.8 or more, more than the kernels of a small call leave time for: compression and attention of 4 heads of 512 tokens
// 14.1 us a pass, 11.1 from here; rotary positions and cache rows of 64 tokens 12.7 us, 5.2 from here.
//
// Every function returns the status of the C entry point, or None where an argument is not what the call takes: the binding then
// goes through its own checks, which say what is wrong.  Nothing is kept from one call to the next.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/l2kv.h"

namespace {

// Entry points of the loaded library, set once by bind().
decltype(&l2kv_decode_attn) decode_attn_entry = nullptr;
decltype(&l2kv_decode_attn_out) decode_attn_out_entry = nullptr;
decltype(&l2kv_compress) compress_entry = nullptr;
decltype(&l2kv_keep_count) keep_count_entry = nullptr;
decltype(&l2kv_rotary_append) rotary_append_entry = nullptr;
decltype(&l2kv_prompt_attn) prompt_attn_entry = nullptr;
decltype(&l2kv_tree_attn) tree_attn_entry = nullptr;
decltype(&l2kv_stream_append_path) append_path_entry = nullptr;
decltype(&l2kv_norm_rotary_append) norm_rotary_append_entry = nullptr;
decltype(&l2kv_paged_append) paged_append_entry = nullptr;
decltype(&l2kv_paged_append_reserved) paged_append_reserved_entry = nullptr;
decltype(&l2kv_paged_attn) paged_attn_entry = nullptr;
decltype(&l2kv_pages_fork) pages_fork_entry = nullptr;
decltype(&l2kv_pages_reserve) pages_reserve_entry = nullptr;
decltype(&l2kv_pages_release) pages_release_entry = nullptr;
decltype(&l2kv_paged_compress) paged_compress_entry = nullptr;

// A plain contiguous device tensor, else nullptr.  (Subclasses of torch.Tensor take the way through Python.)
const at::Tensor* device_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

bool element_type(const at::Tensor& t, l2kv_dtype* dt) {
    const auto s = t.scalar_type();
    *dt = s == at::kFloat ? L2KV_F32 : L2KV_BF16;
    return s == at::kFloat || s == at::kBFloat16;
}

bool number(PyObject* o, double* v) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    *v = PyFloat_AsDouble(o);
    if (*v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

bool integer(PyObject* o, int64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    *v = PyLong_AsLongLong(o);
    if (*v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// The handle of the stream a call goes to, from the binding's own function: only asked for when the arguments are in order.
bool stream_handle(PyObject* stream, PyObject* handle_of, void** handle) {
    PyObject* const v = PyObject_CallFunctionObjArgs(handle_of, stream, nullptr);
    if (v == nullptr) return false;
    *handle = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !(*handle == nullptr && PyErr_Occurred());
}

template <typename F> PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const std::exception&) {           // a tensor without memory, for instance
        Py_RETURN_NONE;
    }
}

template <typename F> PyObject* status_of(F&& call) {
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = (int)call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// (Q, Kc, Vc, O, workspace, scale, stream, stream's handle)
template <bool kAnyOutput> PyObject* decode(PyObject* const* a, Py_ssize_t n_args) {
    const at::Tensor *t[5];
    double scale;
    if (n_args != 8 || !number(a[5], &scale)) Py_RETURN_NONE;
    for (int i = 0; i < 5; ++i)
        if ((t[i] = device_tensor(a[i])) == nullptr) Py_RETURN_NONE;
    const at::Tensor &Q = *t[0], &Kc = *t[1], &Vc = *t[2], &O = *t[3], &ws = *t[4];
    l2kv_dtype dt, out_dt;
    if (Q.dim() != 3 || Kc.dim() != 4 || !element_type(Q, &dt) || !element_type(O, &out_dt)) Py_RETURN_NONE;
    const int64_t B = Q.size(0), Hq = Q.size(1), D = Q.size(2), Hkv = Kc.size(1), n = Kc.size(2);
    if (Kc.size(0) != B || Kc.size(3) != D || Vc.sizes() != Kc.sizes() || Kc.scalar_type() != Q.scalar_type() ||
        Vc.scalar_type() != Q.scalar_type() || O.numel() != B * Hq * D || (!kAnyOutput && out_dt != L2KV_F32))
        Py_RETURN_NONE;
    if (B > INT32_MAX || Hq > INT32_MAX || Hkv > INT32_MAX || D > INT32_MAX) Py_RETURN_NONE;
    const void *q = Q.data_ptr(), *k = Kc.data_ptr(), *v = Vc.data_ptr();
    void *o = O.data_ptr(), *w = ws.data_ptr(), *s;
    const size_t bytes = ws.nbytes();
    if (!stream_handle(a[6], a[7], &s)) return nullptr;
    return status_of([&] {
        if constexpr (kAnyOutput)
            return decode_attn_out_entry(q, k, v, dt, (int32_t)B, (int32_t)Hq, (int32_t)Hkv, n, (int32_t)D, n * D, (float)scale,
                                         out_dt, o, w, bytes, s);
        else
            return decode_attn_entry(q, k, v, dt, (int32_t)B, (int32_t)Hq, (int32_t)Hkv, n, (int32_t)D, n * D, (float)scale,
                                     static_cast<float*>(o), w, bytes, s);
    });
}

PyObject* decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return decode<false>(a, n); }); }
PyObject* decode_attn_out(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return decode<true>(a, n); }); }

// (K, V, norms, kept_idx, Kc, Vc, workspace, keep_ratio, slab_heads, stream, stream's handle)
PyObject* compress_checked(PyObject* const* a, Py_ssize_t n_args) {
    const at::Tensor *t[7];
    double ratio;
    int64_t slab;
    if (n_args != 11 || !number(a[7], &ratio) || !integer(a[8], &slab)) Py_RETURN_NONE;
    for (int i = 0; i < 7; ++i)
        if ((t[i] = device_tensor(a[i])) == nullptr) Py_RETURN_NONE;
    const at::Tensor &K = *t[0], &V = *t[1], &norms = *t[2], &idx = *t[3], &Kc = *t[4], &Vc = *t[5], &ws = *t[6];
    l2kv_dtype dt;
    if (K.dim() < 2 || idx.dim() < 1 || !element_type(K, &dt)) Py_RETURN_NONE;
    const int64_t T = K.size(-2), D = K.size(-1), k = idx.size(-1);
    int64_t n = 1;
    for (int64_t i = 0; i < K.dim() - 2; ++i) n *= K.size(i);
    const auto type = K.scalar_type();
    if (V.sizes() != K.sizes() || V.scalar_type() != type || Kc.scalar_type() != type || Vc.scalar_type() != type ||
        norms.scalar_type() != at::kFloat || norms.numel() != n * T || idx.scalar_type() != at::kInt || idx.numel() != n * k ||
        Kc.numel() != n * k * D || Vc.numel() != n * k * D || D > INT32_MAX)
        Py_RETURN_NONE;
    // The kernels write as many rows as the ratio says, head after head.  (0: no ratio, which the entry point refuses.)
    const int64_t kept = keep_count_entry(T, ratio);
    if (kept > 0 && (k < kept || (k > kept && n > 1))) Py_RETURN_NONE;
    const void *kp = K.data_ptr(), *vp = V.data_ptr();
    float* np = static_cast<float*>(norms.data_ptr());
    int32_t* ip = static_cast<int32_t*>(idx.data_ptr());
    void *kc = Kc.data_ptr(), *vc = Vc.data_ptr(), *w = ws.data_ptr(), *s;
    const size_t bytes = ws.nbytes();
    if (!stream_handle(a[9], a[10], &s)) return nullptr;
    return status_of([&] { return compress_entry(kp, vp, dt, n, T, (int32_t)D, T * D, ratio, slab, np, ip, kc, vc, w, bytes, s); });
}

PyObject* compress(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return compress_checked(a, n); }); }

// The arguments of a call that takes many tensors, one after the other.  `good` falls with the first that is not what the call takes, and
// what is read from then on is not used.
struct Arguments {
    PyObject* const* next;
    bool good = true;

    void require(bool holds) { good = good && holds; }
    bool none() {
        if (*next != Py_None) return false;
        ++next;
        return true;
    }
    const at::Tensor* dense() {
        const at::Tensor* const t = good ? device_tensor(*next) : nullptr;
        ++next;
        require(t != nullptr);
        return t;
    }
    // [tokens, heads, D] whose heads lie side by side, tokens any distance apart: that distance in elements.
    const at::Tensor* tokens(int64_t* stride) {
        PyObject* const o = *next++;
        require(good && THPVariable_CheckExact(o));
        if (!good) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        require(t.is_cuda() && t.dim() == 3 && t.stride(2) == 1 && (t.size(1) <= 1 || t.stride(1) == t.size(2)));
        if (!good) return nullptr;
        *stride = t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2);
        return &t;
    }
    // The memory of a dense tensor of the type and the sizes or the number of elements given.
    template <typename T> T* data(at::ScalarType type, at::IntArrayRef sizes) {
        const at::Tensor* const t = dense();
        require(t != nullptr && t->scalar_type() == type && t->sizes() == sizes);
        return good ? static_cast<T*>(t->data_ptr()) : nullptr;
    }
    template <typename T> T* data(at::ScalarType type, int64_t n) {
        const at::Tensor* const t = dense();
        require(t != nullptr && t->scalar_type() == type && t->numel() == n);
        return good ? static_cast<T*>(t->data_ptr()) : nullptr;
    }
    int32_t* ints(int64_t n) { return data<int32_t>(at::kInt, n); }
    int64_t* longs(int64_t n) { return data<int64_t>(at::kLong, n); }
    int64_t integer() {
        int64_t v = 0;
        require(good && ::integer(*next, &v));
        ++next;
        return v;
    }
    double number() {
        double v = 0;
        require(good && ::number(*next, &v));
        ++next;
        return v;
    }
    void* workspace(size_t* bytes) {
        *bytes = 0;
        if (none()) return nullptr;
        const at::Tensor* const t = dense();
        if (!good) return nullptr;
        *bytes = t->nbytes();
        return t->data_ptr();
    }
    // The stream and the function that gives its handle, the last two.
    bool stream(void** handle) { return stream_handle(next[0], next[1], handle); }
};

bool all_int32(std::initializer_list<int64_t> numbers) {
    for (const int64_t v : numbers)
        if (v < 0 || v > INT32_MAX) return false;
    return true;
}

// Planes [Hkv, rows, D] or caches [B, Hkv, T, D].
struct Planes {
    const void *K = nullptr, *V = nullptr;
    int64_t Hkv = 0, rows = 0, head_stride = 0, D = 0;
};
Planes planes_of(Arguments& a, at::ScalarType type) {
    const at::Tensor *const K = a.dense(), *const V = a.dense();
    Planes p;
    if (!a.good) return p;
    a.require((K->dim() == 3 || K->dim() == 4) && K->scalar_type() == type && V->scalar_type() == type && K->sizes() == V->sizes());
    if (!a.good) return p;
    p = Planes{K->data_ptr(), V->data_ptr(), K->size(-3), K->size(-2), K->size(-2) * K->size(-1), K->size(-1)};
    if (K->dim() == 4) p.rows = ((K->size(0) - 1) * p.Hkv + 1) * K->size(2);
    return p;
}

// (Q, K, V, q_offsets, kv_offsets, kv_lens, max_kv, O, workspace, scale, stream, stream's handle)
PyObject* prompt_attn_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 12) Py_RETURN_NONE;
    Arguments a{args};
    int64_t q_stride = 0;
    l2kv_dtype dt;
    const at::Tensor* const Q = a.tokens(&q_stride);
    if (!a.good || !element_type(*Q, &dt)) Py_RETURN_NONE;
    const auto type = Q->scalar_type();
    const int64_t total = Q->size(0), Hq = Q->size(1), D = Q->size(2);
    const Planes kv = planes_of(a, type);
    const at::Tensor* const q_offsets = a.dense();
    if (!a.good || q_offsets->scalar_type() != at::kLong) Py_RETURN_NONE;
    const int64_t n_seq = q_offsets->numel() - 1;
    const int64_t *const q_off = static_cast<const int64_t*>(q_offsets->data_ptr()), *const kv_off = a.longs(n_seq + 1);
    const int32_t* const lens = a.none() ? nullptr : a.ints(n_seq);
    const int64_t max_kv = a.integer();
    void* const O = a.data<void>(type, Q->sizes());
    size_t bytes;
    void* const ws = a.workspace(&bytes);
    const double scale = a.number();
    a.require(kv.D == D && all_int32({n_seq, Hq, kv.Hkv, D}));
    if (!a.good) Py_RETURN_NONE;
    const void* const q = Q->data_ptr();
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return prompt_attn_entry(q, kv.K, kv.V, dt, (int32_t)n_seq, (int32_t)Hq, (int32_t)kv.Hkv, (int32_t)D, total, q_stride, q_off, kv.rows,
                                 kv.head_stride, kv_off, lens, max_kv, (float)scale, O, ws, bytes, s);
    });
}

// (Q, Kc, Vc, lens, slot_offsets, max_len, Kt, Vt, node_offsets, mask, O, workspace, scale, stream, stream's handle)
PyObject* tree_attn_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 15) Py_RETURN_NONE;
    Arguments a{args};
    int64_t q_stride = 0;
    l2kv_dtype dt;
    const at::Tensor* const Q = a.tokens(&q_stride);
    if (!a.good || !element_type(*Q, &dt)) Py_RETURN_NONE;
    const auto type = Q->scalar_type();
    const int64_t total = Q->size(0), Hq = Q->size(1), D = Q->size(2);
    const Planes kv = planes_of(a, type);
    const at::Tensor* const lens_t = a.dense();
    if (!a.good || lens_t->scalar_type() != at::kInt) Py_RETURN_NONE;
    const int64_t n_seq = lens_t->numel();
    const int32_t* const lens = static_cast<const int32_t*>(lens_t->data_ptr());
    const int64_t* const slot_off = a.longs(n_seq + 1);
    const int64_t max_len = a.integer();
    const int64_t node_sizes[3] = {kv.Hkv, total, D};
    const void *const Kt = a.data<void>(type, at::IntArrayRef(node_sizes)), *const Vt = a.data<void>(type, at::IntArrayRef(node_sizes));
    const int64_t* const node_off = a.longs(n_seq + 1);
    const at::Tensor* const mask = a.dense();
    if (!a.good || mask->dim() != 2 || mask->size(0) != total || mask->scalar_type() != at::kInt) Py_RETURN_NONE;
    const int64_t words = mask->size(1);
    void* const O = a.data<void>(type, Q->sizes());
    size_t bytes;
    void* const ws = a.workspace(&bytes);
    const double scale = a.number();
    a.require(kv.D == D && all_int32({n_seq, Hq, kv.Hkv, D, words}));
    if (!a.good) Py_RETURN_NONE;
    const void* const q = Q->data_ptr();
    const uint32_t* const bits = static_cast<const uint32_t*>(mask->data_ptr());
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return tree_attn_entry(q, kv.K, kv.V, Kt, Vt, dt, (int32_t)n_seq, (int32_t)Hq, (int32_t)kv.Hkv, (int32_t)D, total, q_stride, node_off,
                               bits, (int32_t)words, kv.rows, kv.head_stride, slot_off, lens, max_len, (float)scale, O, ws, bytes, s);
    });
}

// (Q, K, V, positions, freqs, Qr, Kc, Vc, norms_c, pos_c, token_offsets, slot_offsets, lens_in, lens_out, layout, amplitude, stream,
// stream's handle); kNorm: q_weight, k_weight and eps in front of the layout
template <bool kNorm> PyObject* rotary_append_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != (kNorm ? 21 : 18)) Py_RETURN_NONE;
    Arguments a{args};
    int64_t q_stride = 0, k_stride = 0, v_stride = 0, Hq = 0;
    l2kv_dtype dt;
    const at::Tensor* const Q = a.none() ? nullptr : a.tokens(&q_stride);
    const at::Tensor *const K = a.tokens(&k_stride), *const V = a.tokens(&v_stride);
    if (!a.good || !element_type(*K, &dt)) Py_RETURN_NONE;
    const auto type = K->scalar_type();
    const int64_t total = K->size(0), Hkv = K->size(1), D = K->size(2);
    a.require(V->sizes() == K->sizes() && V->scalar_type() == type);
    if (Q != nullptr) {
        Hq = Q->size(1);
        a.require(Q->size(0) == total && Q->size(2) == D && Q->scalar_type() == type);
    }
    const int32_t* const positions = a.ints(total);
    const at::Tensor* const freqs = a.dense();
    if (!a.good || freqs->scalar_type() != at::kDouble) Py_RETURN_NONE;
    void* Qr = nullptr;
    if (!a.none()) {
        if (Q == nullptr) Py_RETURN_NONE;
        Qr = a.data<void>(type, Q->sizes());
    }
    const at::Tensor* const Kc = a.dense();
    if (!a.good || Kc->dim() != 3 || Kc->size(0) != Hkv || Kc->size(2) != D || Kc->scalar_type() != type) Py_RETURN_NONE;
    const int64_t slots = Kc->size(1), row_sizes[2] = {Hkv, slots};
    void* const Vc = a.data<void>(type, Kc->sizes());
    float* const norms = a.data<float>(at::kFloat, at::IntArrayRef(row_sizes));
    int32_t* const pos = a.data<int32_t>(at::kInt, at::IntArrayRef(row_sizes));
    int64_t n_seq = 0;
    const int64_t *token_off = nullptr, *slot_off = nullptr;
    const int32_t* lens_in = nullptr;
    int32_t* lens_out = nullptr;
    if (!a.none()) {
        const at::Tensor* const t = a.dense();
        if (!a.good || t->scalar_type() != at::kLong) Py_RETURN_NONE;
        n_seq = t->numel() - 1;
        token_off = static_cast<const int64_t*>(t->data_ptr());
        if (!a.none()) slot_off = a.longs(n_seq + 1);
        if (!a.none()) lens_in = a.ints(n_seq);
        if (!a.none()) lens_out = a.ints(n_seq);
    } else {
        for (int i = 0; i < 3; ++i) a.require(a.none());
    }
    const float *q_weight = nullptr, *k_weight = nullptr;
    double eps = 0.0;
    if constexpr (kNorm) {
        if (!a.none()) q_weight = a.data<float>(at::kFloat, D);
        if (!a.none()) k_weight = a.data<float>(at::kFloat, D);
        eps = a.number();
    }
    const int64_t layout = a.integer();
    const double amplitude = a.number();
    a.require(all_int32({n_seq, Hq, Hkv, D, 2 * freqs->numel()}) && (layout == L2KV_ROTARY_HALF || layout == L2KV_ROTARY_INTERLEAVED));
    if (!a.good) Py_RETURN_NONE;
    const void *const q = Q == nullptr ? nullptr : Q->data_ptr(), *const k = K->data_ptr(), *const v = V->data_ptr();
    const double* const f = static_cast<const double*>(freqs->data_ptr());
    const int32_t rot_dim = (int32_t)(2 * freqs->numel());
    void *const kc = Kc->data_ptr(), *s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        if constexpr (kNorm)
            return norm_rotary_append_entry(q, k, v, dt, total, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, q_stride, k_stride, v_stride, q_weight, k_weight,
                                            eps, positions, f, rot_dim, (l2kv_rotary_layout)layout, amplitude, (int32_t)n_seq, token_off, slot_off,
                                            lens_in, lens_out, slots, Qr, kc, Vc, norms, pos, s);
        return rotary_append_entry(q, k, v, dt, total, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, q_stride, k_stride, v_stride, positions, f, rot_dim,
                                   (l2kv_rotary_layout)layout, amplitude, (int32_t)n_seq, token_off, slot_off, lens_in, lens_out, slots, Qr, kc,
                                   Vc, norms, pos, s);
    });
}

// (Kt, Vt, norms_t, pos_t, node_offsets, path, path_lens, slot_offsets, lens_in, lens_out, Kc, Vc, norms_c, pos_c, stream, stream's handle)
PyObject* append_path_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 16) Py_RETURN_NONE;
    Arguments a{args};
    l2kv_dtype dt;
    const at::Tensor* const Kt = a.dense();
    if (!a.good || Kt->dim() != 3 || !element_type(*Kt, &dt)) Py_RETURN_NONE;
    const auto type = Kt->scalar_type();
    const int64_t planes = Kt->size(0), total = Kt->size(1), D = Kt->size(2), node_sizes[2] = {planes, total};
    const void* const Vt = a.data<void>(type, Kt->sizes());
    const float* const norms_t = a.data<float>(at::kFloat, at::IntArrayRef(node_sizes));
    const int32_t* const pos_t = a.data<int32_t>(at::kInt, at::IntArrayRef(node_sizes));
    const at::Tensor *const node_offsets = a.dense(), *const path = a.dense();
    if (!a.good || path->dim() != 2 || path->scalar_type() != at::kInt || node_offsets->scalar_type() != at::kLong) Py_RETURN_NONE;
    const int64_t n_seq = path->size(0), max_path = path->size(1);
    a.require(node_offsets->numel() == n_seq + 1);
    const int32_t* const path_lens = a.ints(n_seq);
    const int64_t* const slot_off = a.longs(n_seq + 1);
    const int32_t* const lens_in = a.ints(n_seq);
    int32_t* const lens_out = a.ints(n_seq);
    const at::Tensor* const Kc = a.dense();
    if (!a.good || Kc->dim() != 3 || Kc->size(0) != planes || Kc->size(2) != D || Kc->scalar_type() != type) Py_RETURN_NONE;
    const int64_t slots = Kc->size(1), row_sizes[2] = {planes, slots};
    void* const Vc = a.data<void>(type, Kc->sizes());
    float* const norms = a.data<float>(at::kFloat, at::IntArrayRef(row_sizes));
    int32_t* const pos = a.data<int32_t>(at::kInt, at::IntArrayRef(row_sizes));
    a.require(all_int32({planes, n_seq, D, max_path}));
    if (!a.good) Py_RETURN_NONE;
    const void* const kt = Kt->data_ptr();
    const int64_t* const node_off = static_cast<const int64_t*>(node_offsets->data_ptr());
    const int32_t* const rows = static_cast<const int32_t*>(path->data_ptr());
    void *const kc = Kc->data_ptr(), *s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return append_path_entry(kt, Vt, norms_t, pos_t, dt, (int32_t)planes, (int32_t)n_seq, (int32_t)D, total, node_off, rows, (int32_t)max_path,
                                 path_lens, slot_off, slots, lens_in, lens_out, kc, Vc, norms, pos, s);
    });
}

// A table of pages [n_seq, max_pages].
struct PageTable {
    int32_t* pages = nullptr;
    int64_t n_seq = 0, max_pages = 0;
};
PageTable page_table_of(Arguments& a) {
    const at::Tensor* const t = a.dense();
    a.require(t != nullptr && t->dim() == 2 && t->scalar_type() == at::kInt);
    return a.good ? PageTable{static_cast<int32_t*>(t->data_ptr()), t->size(0), t->size(1)} : PageTable{};
}
// Size of the pages that a cache of so many slots has, and their number.
int64_t page_size_of(Arguments& a, int64_t slots, int64_t* n_pages) {
    const int64_t size = a.integer();
    a.require(size > 0 && size <= INT32_MAX && slots % size == 0);
    *n_pages = a.good ? slots / size : 0;
    return size;
}
// All planes of a cache: Kc, Vc, norms, token ids.
struct Cache {
    l2kv_dtype dt = L2KV_F32;
    void *Kc = nullptr, *Vc = nullptr;
    float* norms = nullptr;
    int32_t* pos = nullptr;
    int64_t planes = 0, slots = 0, D = 0;
};
Cache cache_of(Arguments& a) {
    Cache c;
    const at::Tensor* const K = a.dense();
    a.require(K != nullptr && K->dim() == 3 && element_type(*K, &c.dt));
    if (!a.good) return c;
    c.Kc = K->data_ptr();
    c.planes = K->size(0), c.slots = K->size(1), c.D = K->size(2);
    const int64_t rows[2] = {c.planes, c.slots};
    c.Vc = a.data<void>(K->scalar_type(), K->sizes());
    c.norms = a.data<float>(at::kFloat, at::IntArrayRef(rows));
    c.pos = a.data<int32_t>(at::kInt, at::IntArrayRef(rows));
    return c;
}

// (Q, K, V, positions, freqs, Qr, Kc, Vc, norms_c, pos_c, token_offsets, page_table, page_size, lens_in, lens_out, q_weight, k_weight, eps,
// layout, amplitude, stream, stream's handle); kReserved: ends behind lens_in
template <bool kReserved> PyObject* paged_append_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != (kReserved ? 23 : 22)) Py_RETURN_NONE;
    Arguments a{args};
    int64_t q_stride = 0, k_stride = 0, v_stride = 0, Hq = 0;
    l2kv_dtype dt;
    const at::Tensor* const Q = a.none() ? nullptr : a.tokens(&q_stride);
    const at::Tensor *const K = a.tokens(&k_stride), *const V = a.tokens(&v_stride);
    if (!a.good || !element_type(*K, &dt)) Py_RETURN_NONE;
    const auto type = K->scalar_type();
    const int64_t total = K->size(0), Hkv = K->size(1), D = K->size(2);
    a.require(V->sizes() == K->sizes() && V->scalar_type() == type);
    if (Q != nullptr) {
        Hq = Q->size(1);
        a.require(Q->size(0) == total && Q->size(2) == D && Q->scalar_type() == type);
    }
    const int32_t* const positions = a.ints(total);
    const at::Tensor* const freqs = a.dense();
    if (!a.good || freqs->scalar_type() != at::kDouble) Py_RETURN_NONE;
    void* Qr = nullptr;
    if (!a.none()) {
        if (Q == nullptr) Py_RETURN_NONE;
        Qr = a.data<void>(type, Q->sizes());
    }
    const Cache c = cache_of(a);
    a.require(c.planes == Hkv && c.D == D && c.dt == dt);
    const at::Tensor* const offsets = a.dense();
    const PageTable table = page_table_of(a);
    if (!a.good || offsets->scalar_type() != at::kLong || offsets->numel() != table.n_seq + 1) Py_RETURN_NONE;
    int64_t n_pages;
    const int64_t size = page_size_of(a, c.slots, &n_pages);
    const int32_t* const lens_in = a.ints(table.n_seq);
    const int32_t* ends = nullptr;
    if constexpr (kReserved) {
        if (!a.none()) ends = a.ints(table.n_seq);
    }
    int32_t* const lens_out = a.none() ? nullptr : a.ints(table.n_seq);
    const float* const q_weight = a.none() ? nullptr : a.data<float>(at::kFloat, D);
    const float* const k_weight = a.none() ? nullptr : a.data<float>(at::kFloat, D);
    const double eps = a.number();
    const int64_t layout = a.integer();
    const double amplitude = a.number();
    a.require(all_int32({table.n_seq, table.max_pages, n_pages, Hq, Hkv, D, 2 * freqs->numel()}) &&
              (layout == L2KV_ROTARY_HALF || layout == L2KV_ROTARY_INTERLEAVED));
    if (!a.good) Py_RETURN_NONE;
    const void *const q = Q == nullptr ? nullptr : Q->data_ptr(), *const k = K->data_ptr(), *const v = V->data_ptr();
    const double* const f = static_cast<const double*>(freqs->data_ptr());
    const int32_t rot_dim = (int32_t)(2 * freqs->numel());
    const int64_t* const token_off = static_cast<const int64_t*>(offsets->data_ptr());
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        if constexpr (kReserved)
            return paged_append_reserved_entry(q, k, v, dt, total, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, q_stride, k_stride, v_stride, q_weight, k_weight,
                                               eps, positions, f, rot_dim, (l2kv_rotary_layout)layout, amplitude, (int32_t)table.n_seq, token_off,
                                               table.pages, (int32_t)table.max_pages, (int32_t)size, (int32_t)n_pages, lens_in, ends, lens_out, Qr, c.Kc,
                                               c.Vc, c.norms, c.pos, s);
        return paged_append_entry(q, k, v, dt, total, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, q_stride, k_stride, v_stride, q_weight, k_weight, eps,
                                  positions, f, rot_dim, (l2kv_rotary_layout)layout, amplitude, (int32_t)table.n_seq, token_off, table.pages,
                                  (int32_t)table.max_pages, (int32_t)size, (int32_t)n_pages, lens_in, lens_out, Qr, c.Kc, c.Vc, c.norms, c.pos, s);
    });
}

// (Q, Kc, Vc, q_offsets, page_table, page_size, kv_lens, max_kv, O, workspace, scale, stream, stream's handle)
PyObject* paged_attn_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 13) Py_RETURN_NONE;
    Arguments a{args};
    int64_t q_stride = 0;
    l2kv_dtype dt;
    const at::Tensor* const Q = a.tokens(&q_stride);
    if (!a.good || !element_type(*Q, &dt)) Py_RETURN_NONE;
    const auto type = Q->scalar_type();
    const int64_t total = Q->size(0), Hq = Q->size(1), D = Q->size(2);
    const at::Tensor* const Kc = a.dense();
    if (!a.good || Kc->dim() != 3 || Kc->size(2) != D || Kc->scalar_type() != type) Py_RETURN_NONE;
    const int64_t Hkv = Kc->size(0);
    const void* const Vc = a.data<void>(type, Kc->sizes());
    const at::Tensor* const offsets = a.dense();
    const PageTable table = page_table_of(a);
    if (!a.good || offsets->scalar_type() != at::kLong || offsets->numel() != table.n_seq + 1) Py_RETURN_NONE;
    int64_t n_pages;
    const int64_t size = page_size_of(a, Kc->size(1), &n_pages);
    const int32_t* const lens = a.ints(table.n_seq);
    const int64_t max_kv = a.integer();
    void* const O = a.data<void>(type, Q->sizes());
    size_t bytes;
    void* const ws = a.workspace(&bytes);
    const double scale = a.number();
    a.require(all_int32({table.n_seq, table.max_pages, n_pages, Hq, Hkv, D}));
    if (!a.good) Py_RETURN_NONE;
    const void *const q = Q->data_ptr(), *const k = Kc->data_ptr();
    const int64_t* const q_off = static_cast<const int64_t*>(offsets->data_ptr());
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return paged_attn_entry(q, k, Vc, dt, (int32_t)table.n_seq, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, total, q_stride, q_off, table.pages,
                                (int32_t)table.max_pages, (int32_t)size, (int32_t)n_pages, lens, max_kv, (float)scale, O, ws, bytes, s);
    });
}

// (table_in, lens_in, parents, table_out, lens_out, refs, page_size, stream, stream's handle)
PyObject* pages_fork_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 9) Py_RETURN_NONE;
    Arguments a{args};
    const PageTable in = page_table_of(a);
    const int32_t* const lens_in = a.ints(in.n_seq);
    const at::Tensor* const parents = a.dense();
    const PageTable out = page_table_of(a);
    if (!a.good || parents->scalar_type() != at::kInt || parents->numel() != out.n_seq) Py_RETURN_NONE;
    int32_t* const lens_out = a.ints(out.n_seq);
    const at::Tensor* const refs = a.dense();
    const int64_t size = a.integer();
    a.require(in.max_pages == out.max_pages && all_int32({in.n_seq, out.n_seq, in.max_pages, size}));
    if (!a.good || refs->scalar_type() != at::kInt || refs->numel() > INT32_MAX) Py_RETURN_NONE;
    const int32_t* const from = static_cast<const int32_t*>(parents->data_ptr());
    int32_t* const holders = static_cast<int32_t*>(refs->data_ptr());
    const int32_t n_pages = (int32_t)refs->numel();
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return pages_fork_entry(in.pages, lens_in, (int32_t)in.n_seq, from, (int32_t)out.n_seq, (int32_t)in.max_pages, (int32_t)size, n_pages, out.pages,
                                lens_out, holders, s);
    });
}

// Holders of pages and free ones.
struct Holders {
    int32_t *refs = nullptr, *free_pages = nullptr, *free_count = nullptr;
    int64_t n_pages = 0;
};
Holders holders_of(Arguments& a) {
    Holders h;
    const at::Tensor* const refs = a.dense();
    a.require(refs != nullptr && refs->scalar_type() == at::kInt && refs->numel() <= INT32_MAX);
    if (!a.good) return h;
    h.refs = static_cast<int32_t*>(refs->data_ptr());
    h.n_pages = refs->numel();
    h.free_pages = a.ints(h.n_pages);
    h.free_count = a.ints(1);
    return h;
}

// (page_table, first, to, ends, refs, free_pages, free_count, page_size, Kc, Vc, norms_c, pos_c, workspace, stream, stream's handle)
PyObject* pages_reserve_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 15) Py_RETURN_NONE;
    Arguments a{args};
    const PageTable table = page_table_of(a);
    const int32_t *const from = a.ints(table.n_seq), *const to = a.ints(table.n_seq);
    int32_t* const ends = a.ints(table.n_seq);
    const Holders h = holders_of(a);
    const int64_t size = a.integer();
    const Cache c = cache_of(a);
    size_t bytes;
    void* const ws = a.workspace(&bytes);
    a.require(all_int32({table.n_seq, table.max_pages, size, c.planes, c.D}) && c.slots == h.n_pages * size);
    if (!a.good) Py_RETURN_NONE;
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return pages_reserve_entry(table.pages, (int32_t)table.n_seq, (int32_t)table.max_pages, (int32_t)size, from, to, ends, h.refs, h.free_pages,
                                   h.free_count, (int32_t)h.n_pages, c.dt, (int32_t)c.planes, (int32_t)c.D, c.Kc, c.Vc, c.norms, c.pos, ws, bytes, s);
    });
}

// (page_table, keep_lens, refs, free_pages, free_count, page_size, workspace, stream, stream's handle)
PyObject* pages_release_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 9) Py_RETURN_NONE;
    Arguments a{args};
    const PageTable table = page_table_of(a);
    const int32_t* const keep = a.ints(table.n_seq);
    const Holders h = holders_of(a);
    const int64_t size = a.integer();
    size_t bytes;
    void* const ws = a.workspace(&bytes);
    a.require(all_int32({table.n_seq, table.max_pages, size}));
    if (!a.good) Py_RETURN_NONE;
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return pages_release_entry(table.pages, (int32_t)table.n_seq, (int32_t)table.max_pages, (int32_t)size, keep, h.refs, h.free_pages, h.free_count,
                                   (int32_t)h.n_pages, ws, bytes, s);
    });
}

// (Kc, Vc, norms_c, pos_c, table_in, lens_in, keep, table_out, lens_out, page_size, total_rows, total_kept, max_len, workspace, stream,
// stream's handle)
PyObject* paged_compress_checked(PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 16) Py_RETURN_NONE;
    Arguments a{args};
    const Cache c = cache_of(a);
    const PageTable in = page_table_of(a);
    const int32_t *const lens_in = a.ints(in.n_seq), *const keep = a.ints(in.n_seq);
    const PageTable out = page_table_of(a);
    int32_t* const lens_out = a.ints(in.n_seq);
    int64_t n_pages;
    const int64_t size = page_size_of(a, c.slots, &n_pages), rows = a.integer(), kept = a.integer(), max_len = a.integer();
    size_t bytes;
    void* const ws = a.workspace(&bytes);
    a.require(out.n_seq == in.n_seq && all_int32({in.n_seq, in.max_pages, out.max_pages, n_pages, c.planes, c.D}));
    if (!a.good) Py_RETURN_NONE;
    void* s;
    if (!a.stream(&s)) return nullptr;
    return status_of([&] {
        return paged_compress_entry(c.Kc, c.Vc, c.norms, c.pos, c.dt, (int32_t)c.planes, (int32_t)in.n_seq, (int32_t)c.D, (int32_t)size, (int32_t)n_pages,
                                    in.pages, (int32_t)in.max_pages, lens_in, keep, out.pages, (int32_t)out.max_pages, lens_out, rows, kept, max_len, ws,
                                    bytes, s);
    });
}

PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return paged_append_checked<false>(a, n); }); }
PyObject* paged_append_reserved(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return paged_append_checked<true>(a, n); }); }
PyObject* paged_attn(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return paged_attn_checked(a, n); }); }
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return pages_fork_checked(a, n); }); }
PyObject* pages_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return pages_reserve_checked(a, n); }); }
PyObject* pages_release(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return pages_release_checked(a, n); }); }
PyObject* paged_compress(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return paged_compress_checked(a, n); }); }
PyObject* prompt_attn(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return prompt_attn_checked(a, n); }); }
PyObject* tree_attn(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return tree_attn_checked(a, n); }); }
PyObject* rotary_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return rotary_append_checked<false>(a, n); }); }
PyObject* norm_rotary_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return rotary_append_checked<true>(a, n); }); }
PyObject* append_path(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded([&] { return append_path_checked(a, n); }); }

PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long attn, attn_out, comp, count, rotary, prompt, tree, path, append, paged, fork, reserve, release, compact, norm, reserved;
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKKKKK", &attn, &attn_out, &comp, &count, &rotary, &prompt, &tree, &path, &append, &paged, &fork, &reserve,
                          &release, &compact, &norm, &reserved))
        return nullptr;
    norm_rotary_append_entry = reinterpret_cast<decltype(norm_rotary_append_entry)>(norm);
    paged_append_entry = reinterpret_cast<decltype(paged_append_entry)>(append);
    paged_append_reserved_entry = reinterpret_cast<decltype(paged_append_reserved_entry)>(reserved);
    paged_attn_entry = reinterpret_cast<decltype(paged_attn_entry)>(paged);
    pages_fork_entry = reinterpret_cast<decltype(pages_fork_entry)>(fork);
    pages_reserve_entry = reinterpret_cast<decltype(pages_reserve_entry)>(reserve);
    pages_release_entry = reinterpret_cast<decltype(pages_release_entry)>(release);
    paged_compress_entry = reinterpret_cast<decltype(paged_compress_entry)>(compact);
    rotary_append_entry = reinterpret_cast<decltype(rotary_append_entry)>(rotary);
    prompt_attn_entry = reinterpret_cast<decltype(prompt_attn_entry)>(prompt);
    tree_attn_entry = reinterpret_cast<decltype(tree_attn_entry)>(tree);
    append_path_entry = reinterpret_cast<decltype(append_path_entry)>(path);
    decode_attn_entry = reinterpret_cast<decltype(decode_attn_entry)>(attn);
    decode_attn_out_entry = reinterpret_cast<decltype(decode_attn_out_entry)>(attn_out);
    compress_entry = reinterpret_cast<decltype(compress_entry)>(comp);
    keep_count_entry = reinterpret_cast<decltype(keep_count_entry)>(count);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"decode_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_attn)), METH_FASTCALL, nullptr},
                         {"decode_attn_out", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_attn_out)), METH_FASTCALL, nullptr},
                         {"compress", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(compress)), METH_FASTCALL, nullptr},
                         {"rotary_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary_append)), METH_FASTCALL, nullptr},
                         {"prompt_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prompt_attn)), METH_FASTCALL, nullptr},
                         {"tree_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(tree_attn)), METH_FASTCALL, nullptr},
                         {"append_path", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append_path)), METH_FASTCALL, nullptr},
                         {"norm_rotary_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(norm_rotary_append)), METH_FASTCALL, nullptr},
                         {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append)), METH_FASTCALL, nullptr},
                         {"paged_append_reserved", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append_reserved)), METH_FASTCALL, nullptr},
                         {"paged_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attn)), METH_FASTCALL, nullptr},
                         {"pages_fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(pages_fork)), METH_FASTCALL, nullptr},
                         {"pages_reserve", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(pages_reserve)), METH_FASTCALL, nullptr},
                         {"pages_release", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(pages_release)), METH_FASTCALL, nullptr},
                         {"paged_compress", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_compress)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "l2kv_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_l2kv_calls() {
    PyObject* const m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", L2KV_TORCH) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
