// Argument marshalling of the calls that a program makes once per layer and token, in C++: what binding.py's wrappers check and pass on,
// read straight from the tensors.  A call that is anything but ordinary (an output to allocate, a tensor subclass, a layout or a type that
// the wrappers refuse) is left to them: every function returns the library's status, or -1 for "not taken", with nothing done.
//
// Bound by the library's launch.  The wrappers' attribute look-ups and ctypes' conversions (some twenty of each a call) took as long again: host
// time of a decode call with a tail 9.7 us, 6.3 so, of two launches for several query rows 13.3 and 8.6.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <type_traits>

#include "../../include/semanticache.h"

namespace {

constexpr int kNotTaken = -1;

// A tensor argument: `t` is NULL for None.  False: not a plain tensor on the GPU.
inline bool take(PyObject *o, const at::Tensor *&t) {
    t = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    t = &THPVariable_Unpack(o);
    return t->is_cuda();
}
inline bool take_some(PyObject *o, const at::Tensor *&t) { return take(o, t) && t != nullptr; }
// whether the others live where `t` does
template <typename... T> inline bool beside(const at::Tensor *t, const T *...others) {
    const auto d = t->get_device();
    return ((!others || others->get_device() == d) && ...);
}
inline int code(const at::Tensor &t) {
    switch (t.scalar_type()) {
        case at::kFloat: return SC_F32;
        case at::kBFloat16: return SC_BF16;
        default: return -1;
    }
}
inline void *data(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
template <typename T> inline T *data(const at::Tensor *t) { return static_cast<T *>(data(t)); }

inline void *pointer(PyObject *o) { return PyLong_AsVoidPtr(o); }

// The call itself runs without the interpreter lock, as under ctypes.
template <typename F> inline int unlocked(F f) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return status;
}
// A tensor without storage (or anything else that throws) is left to the wrapper, which raises its own error.
template <typename F> PyObject *guarded(F f) {
    int status;
    try {
        status = f();
    } catch (...) {
        status = kNotTaken;
    }
    if (PyErr_Occurred()) {
        if (status != kNotTaken) return nullptr;
        PyErr_Clear();
    }
    return PyLong_FromLong(status);
}

struct Cache {      // Kc, Vc, counts, comp_lens and, if any, Kt, Vt, tail_lens
    const at::Tensor *Kc, *Vc, *counts, *lens, *Kt, *Vt, *tail_lens;
    int kv_code, Hkv, cap, tail_cap;
    bool read(PyObject *const *a, PyObject *const *tail, int64_t d) {
        if (!take_some(a[0], Kc) || !take_some(a[1], Vc) || !take_some(a[2], counts) || !take_some(a[3], lens)) return false;
        if (Kc->dim() != 4 || !Kc->is_contiguous() || !Vc->is_contiguous() || !counts->is_contiguous() || !lens->is_contiguous()) return false;
        kv_code = code(*Kc);
        Hkv = (int)Kc->size(1);
        cap = (int)Kc->size(2);
        tail_cap = 0;
        if (tail[0] == Py_None) {
            Kt = Vt = tail_lens = nullptr;
            return kv_code >= 0;
        }
        if (!take_some(tail[0], Kt) || !take_some(tail[1], Vt) || !take_some(tail[2], tail_lens)) return false;
        if (Kt->dim() != 4 || Kt->sizes() != Vt->sizes() || Kt->scalar_type() != Kc->scalar_type() || Vt->scalar_type() != Kc->scalar_type()) return false;
        if (Kt->size(0) != Kc->size(0) || Kt->size(1) != Kc->size(1) || Kt->size(3) != d) return false;
        tail_cap = (int)Kt->size(2);
        return kv_code >= 0 && Kt->is_contiguous() && Vt->is_contiguous() && tail_lens->is_contiguous();
    }
};

// (mask, seq_lens, offsets, num_chunks, stream)
PyObject *segment(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *mask, *seq_lens, *offsets, *num_chunks;
        if (n != 5 || !take_some(a[0], mask) || !take(a[1], seq_lens) || !take_some(a[2], offsets) || !take_some(a[3], num_chunks)) return kNotTaken;
        if (mask->scalar_type() != at::kByte || mask->dim() != 2 || mask->stride(1) != 1 || offsets->dim() != 2) return kNotTaken;
        void *stream = pointer(a[4]);
        const auto *m = data<const uint8_t>(mask);
        const auto *sl = data<const int32_t>(seq_lens);
        auto *off = data<int32_t>(offsets), *nch = data<int32_t>(num_chunks);
        return unlocked([&]() {
            return (int)sc_segment(m, mask->stride(0), sl, (int)mask->size(0), (int)mask->size(1), off, offsets->stride(0), (int)offsets->size(1), nch, nullptr, 0, stream);
        });
    });
}

// (K, V, offsets, num_chunks, tau, seq_lens, cap, Kc, Vc, counts, comp_lens, cluster_id, base_lens, workspace, bytes, stream)
PyObject *merge(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *K, *V, *offsets, *num_chunks, *seq_lens, *Kc, *Vc, *counts, *lens, *ids, *base;
        if (n != 16 || !take_some(a[0], K) || !take_some(a[1], V) || !take_some(a[2], offsets) || !take(a[3], num_chunks) || !take(a[5], seq_lens)) return kNotTaken;
        if (!take_some(a[7], Kc) || !take_some(a[8], Vc) || !take_some(a[9], counts) || !take_some(a[10], lens) || !take(a[11], ids) || !take(a[12], base))
            return kNotTaken;
        if (K->dim() != 4 || K->sizes() != V->sizes() || K->strides() != V->strides() || K->stride(3) != 1 || K->scalar_type() != V->scalar_type()) return kNotTaken;
        if (!Kc->is_contiguous() || !Vc->is_contiguous() || !counts->is_contiguous() || !lens->is_contiguous()) return kNotTaken;
        const double tau = PyFloat_AsDouble(a[4]);
        const long cap = PyLong_AsLong(a[6]);
        const size_t bytes = PyLong_AsSize_t(a[14]);
        void *w = pointer(a[13]), *stream = pointer(a[15]);
        const int in = code(*K), out = code(*Kc);
        if (PyErr_Occurred() || in < 0 || out < 0 || cap != (int)cap || offsets->dim() < 1) return kNotTaken;
        if (base && (Kc->dim() != 4 || Kc->size(2) != cap || !base->is_contiguous())) return kNotTaken;
        const void *k = data(K), *v = data(V);
        const auto *sl = data<const int32_t>(seq_lens), *off = data<const int32_t>(offsets), *nch = data<const int32_t>(num_chunks), *bl = data<const int32_t>(base);
        void *kc = data(Kc), *vc = data(Vc);
        auto *cnt = data<int32_t>(counts), *cl = data<int32_t>(lens), *cid = data<int32_t>(ids);
        const int B = (int)K->size(0), H = (int)K->size(1), N = (int)K->size(2), d = (int)K->size(3);
        return unlocked([&]() {
            if (base)
                return (int)sc_gsc_merge_append(k, v, (sc_dtype)in, K->stride(0), K->stride(1), K->stride(2), sl, off, offsets->stride(0), nch, B, H, N, d, (float)tau,
                                                kc, vc, (sc_dtype)out, (int)cap, cnt, bl, cl, cid, w, bytes, stream);
            return (int)sc_gsc_merge(k, v, (sc_dtype)in, K->stride(0), K->stride(1), K->stride(2), sl, off, offsets->stride(0), nch, B, H, N, d, (float)tau, kc, vc,
                                     (sc_dtype)out, (int)cap, cnt, cl, cid, w, bytes, stream);
        });
    });
}

// (Q, Kc, Vc, counts, comp_lens, scale, O, lse, Kt, Vt, tail_lens, workspace, bytes, stream)
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *Q, *O, *lse;
        Cache c;
        if (n != 14 || !take_some(a[0], Q) || Q->dim() != 3 || !Q->is_contiguous()) return kNotTaken;
        const int B = (int)Q->size(0), Hq = (int)Q->size(1), d = (int)Q->size(2);
        if (!c.read(a + 1, a + 8, d) || !take_some(a[6], O) || !take(a[7], lse)) return kNotTaken;
        const double scale = PyFloat_AsDouble(a[5]);
        const size_t bytes = PyLong_AsSize_t(a[12]);
        void *w = pointer(a[11]), *stream = pointer(a[13]);
        const int qc = code(*Q), oc = code(*O);
        if (PyErr_Occurred() || qc < 0 || oc < 0) return kNotTaken;
        const void *q = data(Q), *kc = data(c.Kc), *vc = data(c.Vc), *kt = data(c.Kt), *vt = data(c.Vt);
        const auto *cnt = data<const int32_t>(c.counts), *cl = data<const int32_t>(c.lens), *tl = data<const int32_t>(c.tail_lens);
        void *o = data(O);
        auto *l = data<float>(lse);
        return unlocked([&]() {
            if (c.Kt)
                return (int)sc_decode_attn_tail(q, (sc_dtype)qc, kc, vc, (sc_dtype)c.kv_code, c.cap, cnt, cl, kt, vt, c.tail_cap, tl, B, Hq, c.Hkv, d, (float)scale, o,
                                                (sc_dtype)oc, l, w, bytes, stream);
            return (int)sc_decode_attn(q, (sc_dtype)qc, kc, vc, (sc_dtype)c.kv_code, c.cap, cnt, cl, B, Hq, c.Hkv, d, (float)scale, o, (sc_dtype)oc, l, w, bytes, stream);
        });
    });
}

// (Q, Kc, Vc, counts, comp_lens, scale, O, lse, Kt, Vt, tail_lens, causal, workspace, bytes, stream)
PyObject *multi(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *Q, *O, *lse;
        Cache c;
        if (n != 15 || !take_some(a[0], Q) || Q->dim() != 4 || !Q->is_contiguous()) return kNotTaken;
        const int nq = (int)Q->size(0), B = (int)Q->size(1), Hq = (int)Q->size(2), d = (int)Q->size(3);
        if (!c.read(a + 1, a + 8, d) || !take_some(a[6], O) || !take(a[7], lse)) return kNotTaken;
        const double scale = PyFloat_AsDouble(a[5]);
        const int causal = PyObject_IsTrue(a[11]);
        const size_t bytes = PyLong_AsSize_t(a[13]);
        void *w = pointer(a[12]), *stream = pointer(a[14]);
        const int qc = code(*Q), oc = code(*O);
        if (PyErr_Occurred() || qc < 0 || oc < 0) return kNotTaken;
        const void *q = data(Q), *kc = data(c.Kc), *vc = data(c.Vc), *kt = data(c.Kt), *vt = data(c.Vt);
        const auto *cnt = data<const int32_t>(c.counts), *cl = data<const int32_t>(c.lens), *tl = data<const int32_t>(c.tail_lens);
        void *o = data(O);
        auto *l = data<float>(lse);
        return unlocked([&]() {
            if (c.Kt)
                return (int)sc_multi_attn_tail(q, (sc_dtype)qc, nq, kc, vc, (sc_dtype)c.kv_code, c.cap, cnt, cl, kt, vt, c.tail_cap, tl, causal, B, Hq, c.Hkv, d,
                                               (float)scale, o, (sc_dtype)oc, l, w, bytes, stream);
            return (int)sc_multi_attn(q, (sc_dtype)qc, nq, kc, vc, (sc_dtype)c.kv_code, c.cap, cnt, cl, B, Hq, c.Hkv, d, (float)scale, o, (sc_dtype)oc, l, w, bytes, stream);
        });
    });
}

// ---- a cache held in pages: the first argument is the address of its sc_paged_cache, which the wrapper keeps
inline bool is_i32(const at::Tensor *t) { return t->scalar_type() == at::kInt && t->is_contiguous(); }
// lengths [B] or [B, Hkv]
template <typename C> inline bool lengths(const at::Tensor *t, const C *c, bool &per_head) {
    if (!is_i32(t) || t->dim() < 1 || t->dim() > 2 || t->size(0) != c->B) return false;
    per_head = t->dim() == 2;
    return !per_head || t->size(1) == c->Hkv;
}
inline bool is_shape(const at::Tensor *t, int64_t a, int64_t b, int64_t c) { return t->dim() == 3 && t->size(0) == a && t->size(1) == b && t->size(2) == c; }

inline int dtype_of(const sc_paged_cache *c) { return c->dtype; }
inline int dtype_of(const sc_paged8_cache *) { return -1; }
inline sc_status append_to(const sc_paged_cache *c, const sc_paged_rows *r, int, void *stream) { return sc_paged_append(c, r, stream); }
inline sc_status append_to(const sc_paged8_cache *c, const sc_paged_rows *r, int code, void *stream) { return sc_paged8_append(c, r, (sc_dtype)code, stream); }

// (cache, K, V, base_lens, lens, new_lens, counts, Q, Q_out, cos_sin, positions, interleaved, stream)
template <typename C> PyObject *append(PyObject *const *a, Py_ssize_t n) {
    constexpr bool codes = std::is_same<C, sc_paged8_cache>::value;
    return guarded([&]() {
        const at::Tensor *K, *V, *base, *lens, *fresh, *counts, *Q, *Qo, *angles, *positions;
        if (n != 13 || !take_some(a[1], K) || !take_some(a[2], V) || !take_some(a[3], base) || !take_some(a[4], lens) || !take(a[5], fresh) || !take(a[6], counts)) return kNotTaken;
        if (!take(a[7], Q) || !take(a[8], Qo) || !take(a[9], angles) || !take(a[10], positions)) return kNotTaken;
        if (codes && !beside(K, V, base, lens, fresh, counts, Q, Qo, angles, positions)) return kNotTaken;
        const auto *c = static_cast<const C *>(pointer(a[0]));
        const int turned = PyObject_IsTrue(a[11]);
        void *stream = pointer(a[12]);
        if (PyErr_Occurred() || !c) return kNotTaken;
        bool per_head, same;
        if (K->dim() != 4 || K->sizes() != V->sizes() || K->size(0) != c->B || K->size(1) != c->Hkv || K->size(3) != c->d) return kNotTaken;
        if (code(*K) < 0 || code(*K) != code(*V) || (!codes && code(*K) != dtype_of(c)) || K->stride(3) != 1 || V->stride(3) != 1) return kNotTaken;
        if (!lengths(base, c, per_head) || !lengths(lens, c, same) || same != per_head) return kNotTaken;
        if (fresh && (!lengths(fresh, c, same) || same != per_head)) return kNotTaken;
        const int64_t N = K->size(2);
        if (N != (int)N || (counts && (!is_i32(counts) || !is_shape(counts, c->B, c->Hkv, N)))) return kNotTaken;
        if (angles && (angles->dim() != 2 || angles->scalar_type() != at::kFloat || !angles->is_contiguous() || angles->size(0) != (int)angles->size(0))) return kNotTaken;
        if (positions && (!is_i32(positions) || positions->dim() != 1 || positions->size(0) != c->B)) return kNotTaken;
        sc_paged_rows r = {};
        r.K = data(K); r.V = data(V);
        r.k_stride_b = K->stride(0); r.k_stride_h = K->stride(1); r.k_stride_n = K->stride(2);
        r.v_stride_b = V->stride(0); r.v_stride_h = V->stride(1); r.v_stride_n = V->stride(2);
        r.counts = data<const int32_t>(counts);
        r.N = (int)N; r.per_head = per_head;
        r.base_lens = data<const int32_t>(base); r.new_lens = data<const int32_t>(fresh); r.lens = data<int32_t>(lens);
        r.cos_sin = data<const float>(angles); r.positions = data<const int32_t>(positions); r.interleaved = turned;
        if (angles) { r.max_position = (int)angles->size(0); r.rot = (int)angles->size(1); }
        if (Q) {
            if (!Qo || Q->dim() != 4 || Q->sizes() != Qo->sizes() || Q->size(0) != c->B || Q->size(2) != N || Q->size(3) != c->d) return kNotTaken;
            if (code(*Q) < 0 || Q->scalar_type() != Qo->scalar_type() || Q->stride(3) != 1 || Qo->stride(3) != 1) return kNotTaken;
            r.Q = data(Q); r.Q_out = data(Qo); r.Hq = (int)Q->size(1); r.q_dtype = code(*Q);
            r.q_stride_b = Q->stride(0); r.q_stride_h = Q->stride(1); r.q_stride_n = Q->stride(2);
            r.o_stride_b = Qo->stride(0); r.o_stride_h = Qo->stride(1); r.o_stride_n = Qo->stride(2);
        }
        return unlocked([&]() { return (int)append_to(c, &r, code(*K), stream); });
    });
}
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) { return append<sc_paged_cache>(a, n); }
PyObject *paged8_append(PyObject *, PyObject *const *a, Py_ssize_t n) { return append<sc_paged8_cache>(a, n); }

// (cache, Q, lens, scale, O, lse, sel, sel_lens, workspace, bytes, stream)
PyObject *paged_decode(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *Q, *lens, *O, *lse, *sel, *many;
        if (n != 11 || !take_some(a[1], Q) || !take_some(a[2], lens) || !take_some(a[4], O) || !take(a[5], lse) || !take(a[6], sel) || !take(a[7], many)) return kNotTaken;
        const auto *c = static_cast<const sc_paged_cache *>(pointer(a[0]));
        const double scale = PyFloat_AsDouble(a[3]);
        const size_t bytes = PyLong_AsSize_t(a[9]);
        void *w = pointer(a[8]), *stream = pointer(a[10]);
        if (PyErr_Occurred() || !c) return kNotTaken;
        bool per_head;
        if (Q->dim() != 3 || Q->size(0) != c->B || Q->size(2) != c->d || !Q->is_contiguous() || Q->sizes() != O->sizes() || !O->is_contiguous()) return kNotTaken;
        const int qc = code(*Q), oc = code(*O);
        if (qc < 0 || oc < 0 || !lengths(lens, c, per_head)) return kNotTaken;
        if (lse && (lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != c->B || lse->size(1) != Q->size(1) || !lse->is_contiguous())) return kNotTaken;
        if (!sel != !many) return kNotTaken;
        if (sel && (!is_i32(sel) || sel->dim() != 3 || sel->size(0) != c->B || sel->size(1) != c->Hkv || sel->size(2) != (int)sel->size(2))) return kNotTaken;
        if (sel && (!is_i32(many) || many->dim() != 2 || many->size(0) != c->B || many->size(1) != c->Hkv)) return kNotTaken;
        const void *q = data(Q);
        const auto *l = data<const int32_t>(lens), *s = data<const int32_t>(sel), *m = data<const int32_t>(many);
        void *o = data(O);
        auto *e = data<float>(lse);
        return unlocked([&]() {
            return (int)sc_paged_decode_attn(c, q, (sc_dtype)qc, (int)Q->size(1), l, per_head, s, m, sel ? (int)sel->size(2) : 0, (float)scale, o, (sc_dtype)oc, e, w, bytes, stream);
        });
    });
}

// (cache, Q, lens, keep, first, recent, sel, sel_lens, workspace, bytes, stream)
PyObject *paged_select(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *Q, *lens, *sel, *many;
        if (n != 11 || !take_some(a[1], Q) || !take_some(a[2], lens) || !take_some(a[6], sel) || !take_some(a[7], many)) return kNotTaken;
        const auto *c = static_cast<const sc_paged_cache *>(pointer(a[0]));
        const long keep = PyLong_AsLong(a[3]), first = PyLong_AsLong(a[4]), recent = PyLong_AsLong(a[5]);
        const size_t bytes = PyLong_AsSize_t(a[9]);
        void *w = pointer(a[8]), *stream = pointer(a[10]);
        if (PyErr_Occurred() || !c || keep != (int)keep || first != (int)first || recent != (int)recent) return kNotTaken;
        bool per_head;
        if (Q->dim() != 3 || Q->size(0) != c->B || Q->size(2) != c->d || !Q->is_contiguous() || code(*Q) < 0 || !lengths(lens, c, per_head)) return kNotTaken;
        if (!is_i32(sel) || !is_shape(sel, c->B, c->Hkv, keep) || !is_i32(many) || many->dim() != 2 || many->size(0) != c->B || many->size(1) != c->Hkv) return kNotTaken;
        const void *q = data(Q);
        const auto *l = data<const int32_t>(lens);
        auto *s = data<int32_t>(sel), *m = data<int32_t>(many);
        return unlocked([&]() {
            return (int)sc_paged_select(c, q, (sc_dtype)code(*Q), (int)Q->size(1), l, per_head, (int)keep, (int)first, (int)recent, s, m, w, bytes, stream);
        });
    });
}

// (cache, Q, lens, window, sinks, scale, O, lse, workspace, bytes, stream)
template <typename C, typename F> PyObject *windowed(PyObject *const *a, Py_ssize_t n, F attend) {
    return guarded([&]() {
        const at::Tensor *Q, *lens, *O, *lse;
        if (n != 11 || !take_some(a[1], Q) || !take_some(a[2], lens) || !take_some(a[6], O) || !take(a[7], lse) || !beside(Q, lens, O, lse)) return kNotTaken;
        const auto *c = static_cast<const C *>(pointer(a[0]));
        const long window = PyLong_AsLong(a[3]), sinks = PyLong_AsLong(a[4]);
        const double scale = PyFloat_AsDouble(a[5]);
        const size_t bytes = PyLong_AsSize_t(a[9]);
        void *w = pointer(a[8]), *stream = pointer(a[10]);
        if (PyErr_Occurred() || !c || window != (int)window || sinks != (int)sinks) return kNotTaken;
        bool per_head;
        if (Q->dim() != 3 || Q->size(0) != c->B || Q->size(2) != c->d || !Q->is_contiguous() || Q->sizes() != O->sizes() || !O->is_contiguous()) return kNotTaken;
        const int qc = code(*Q), oc = code(*O);
        if (qc < 0 || oc < 0 || Q->size(1) != (int)Q->size(1) || !lengths(lens, c, per_head)) return kNotTaken;
        if (lse && (lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != c->B || lse->size(1) != Q->size(1) || !lse->is_contiguous())) return kNotTaken;
        const void *q = data(Q);
        const auto *l = data<const int32_t>(lens);
        void *o = data(O);
        auto *e = data<float>(lse);
        return unlocked([&]() {
            return (int)attend(c, q, (sc_dtype)qc, (int)Q->size(1), l, per_head, (int)window, (int)sinks, (float)scale, o, (sc_dtype)oc, e, w, bytes, stream);
        });
    });
}
PyObject *paged_window(PyObject *, PyObject *const *a, Py_ssize_t n) { return windowed<sc_paged_cache>(a, n, sc_paged_window_attn); }
PyObject *paged8_decode(PyObject *, PyObject *const *a, Py_ssize_t n) { return windowed<sc_paged8_cache>(a, n, sc_paged8_decode_attn); }

// (table, page_rows, base_lens, lens, free_pages, num_free, new_lens, N, window, sinks, slots, workspace, bytes, stream)
PyObject *paged_reserve(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *table, *base, *lens, *free_pages, *num_free, *fresh, *slots;
        if (n != 14 || !take_some(a[0], table) || !take_some(a[2], base) || !take_some(a[3], lens) || !take_some(a[4], free_pages) || !take_some(a[5], num_free)) return kNotTaken;
        if (!take(a[6], fresh) || !take(a[10], slots) || !beside(table, base, lens, free_pages, num_free, fresh, slots)) return kNotTaken;
        const long rows = PyLong_AsLong(a[1]), N = PyLong_AsLong(a[7]), window = PyLong_AsLong(a[8]), sinks = PyLong_AsLong(a[9]);
        const size_t bytes = PyLong_AsSize_t(a[12]);
        void *w = pointer(a[11]), *stream = pointer(a[13]);
        if (PyErr_Occurred() || rows != (int)rows || N != (int)N || window != (int)window || sinks != (int)sinks) return kNotTaken;
        const int64_t dims = table->dim();
        if (dims < 2 || !is_i32(table) || !is_i32(base) || !is_i32(lens) || (fresh && !is_i32(fresh)) || (slots && !is_i32(slots))) return kNotTaken;
        const auto shape = table->sizes().slice(0, dims - 1);
        if (base->sizes() != shape || lens->sizes() != shape || (fresh && fresh->sizes() != shape)) return kNotTaken;
        if (slots && (slots->dim() != dims || slots->sizes().slice(0, dims - 1) != shape || slots->size(dims - 1) != N)) return kNotTaken;
        if (!is_i32(free_pages) || free_pages->dim() != 1 || !is_i32(num_free) || num_free->dim() != 1 || num_free->size(0) != 1) return kNotTaken;
        const int64_t S = base->numel(), P = table->size(dims - 1), pages = free_pages->size(0);
        if (S != (int)S || P != (int)P || pages != (int)pages) return kNotTaken;
        auto *t = data<int32_t>(table), *l = data<int32_t>(lens), *f = data<int32_t>(free_pages), *m = data<int32_t>(num_free), *sl = data<int32_t>(slots);
        const auto *b = data<const int32_t>(base), *nw = data<const int32_t>(fresh);
        return unlocked([&]() {
            return (int)sc_paged_reserve(t, (int)S, (int)P, (int)pages, (int)rows, b, nw, (int)N, (int)window, (int)sinks, f, m, l, sl, w, bytes, stream);
        });
    });
}

// (Q, K, V, q_lens, kv_lens, window, sinks, scale, O, lse, workspace, bytes, stream)
PyObject *prompt(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() {
        const at::Tensor *Q, *K, *V, *O, *ql, *kl, *lse;
        if (n != 13 || !take_some(a[0], Q) || !take_some(a[1], K) || !take_some(a[2], V) || !take(a[3], ql) || !take(a[4], kl) || !take_some(a[8], O) || !take(a[9], lse)) return kNotTaken;
        if (!beside(Q, K, V, ql, kl, O, lse)) return kNotTaken;
        const long window = PyLong_AsLong(a[5]), sinks = PyLong_AsLong(a[6]);
        const double scale = PyFloat_AsDouble(a[7]);
        const size_t bytes = PyLong_AsSize_t(a[11]);
        void *w = pointer(a[10]), *stream = pointer(a[12]);
        if (PyErr_Occurred() || window != (int)window || sinks != (int)sinks) return kNotTaken;
        if (Q->dim() != 4 || K->dim() != 4 || K->sizes() != V->sizes() || K->size(0) != Q->size(0) || K->size(3) != Q->size(3) || Q->sizes() != O->sizes()) return kNotTaken;
        if (code(*Q) < 0 || code(*K) != code(*Q) || code(*V) != code(*Q) || code(*O) != code(*Q)) return kNotTaken;
        if (Q->stride(3) != 1 || K->stride(3) != 1 || V->stride(3) != 1 || O->stride(3) != 1) return kNotTaken;
        for (int i = 0; i < 4; ++i)
            if (Q->size(i) != (int)Q->size(i) || K->size(i) != (int)K->size(i)) return kNotTaken;
        const int64_t B = Q->size(0);
        if (ql && (!is_i32(ql) || ql->dim() != 1 || ql->size(0) != B)) return kNotTaken;
        if (kl && (!is_i32(kl) || kl->dim() != 1 || kl->size(0) != B)) return kNotTaken;
        if (lse && (lse->scalar_type() != at::kFloat || !is_shape(lse, B, Q->size(1), Q->size(2)) || !lse->is_contiguous())) return kNotTaken;
        sc_prompt x = {};
        x.Q = data(Q); x.K = data(K); x.V = data(V); x.O = data(O); x.lse = data<float>(lse);
        x.q_stride_b = Q->stride(0); x.q_stride_h = Q->stride(1); x.q_stride_n = Q->stride(2);
        x.k_stride_b = K->stride(0); x.k_stride_h = K->stride(1); x.k_stride_n = K->stride(2);
        x.v_stride_b = V->stride(0); x.v_stride_h = V->stride(1); x.v_stride_n = V->stride(2);
        x.o_stride_b = O->stride(0); x.o_stride_h = O->stride(1); x.o_stride_n = O->stride(2);
        x.q_lens = data<const int32_t>(ql); x.kv_lens = data<const int32_t>(kl);
        x.dtype = code(*Q);
        x.B = (int)B; x.Hq = (int)Q->size(1); x.Hkv = (int)K->size(1); x.N = (int)Q->size(2); x.M = (int)K->size(2); x.d = (int)Q->size(3);
        x.window = (int)window; x.sinks = (int)sinks; x.scale = (float)scale;
        return unlocked([&]() { return (int)sc_prompt_attn(&x, w, bytes, stream); });
    });
}

PyMethodDef methods[] = {
    {"segment", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(segment)), METH_FASTCALL, nullptr},
    {"merge", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(merge)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode)), METH_FASTCALL, nullptr},
    {"multi", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(multi)), METH_FASTCALL, nullptr},
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append)), METH_FASTCALL, nullptr},
    {"paged_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_decode)), METH_FASTCALL, nullptr},
    {"paged_select", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_select)), METH_FASTCALL, nullptr},
    {"paged8_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged8_append)), METH_FASTCALL, nullptr},
    {"paged_window", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_window)), METH_FASTCALL, nullptr},
    {"paged8_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged8_decode)), METH_FASTCALL, nullptr},
    {"paged_reserve", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_reserve)), METH_FASTCALL, nullptr},
    {"prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prompt)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch that the tensors' layout is known from; the loader compares it with the one at hand
PyMODINIT_FUNC PyInit__native() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", SC_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
