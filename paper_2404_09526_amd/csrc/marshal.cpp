// The argument checks of binding.py's calls, in native code, for the calls a serving loop makes step after step: everything given (outputs,
// workspace), plain tensors on the device, plain numbers.  Each function checks what the Python beside it checks, calls the C ABI
// and returns its status; for anything else it does nothing and returns None, and the Python goes through the same checks
// one by one and says what is wrong (or takes what is not plain).  What bounds a step of few short requests is the host:
// appended and decoded with three peers, 4 requests, the two calls took 9.4 us of Python beside 10 us in the library and the runtime.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>

#include "esp.h"

namespace {

PyObject* g_stream = nullptr;                      // binding._stream
PyObject* g_device = nullptr;                      // the number of the current device
decltype(&esp_kv_append) p_append;
decltype(&esp_partial_attn_decode) p_decode;
decltype(&esp_partial_attn_decode_merge) p_decode_merge;
decltype(&esp_partial_attn_prefill) p_prefill;
decltype(&esp_partial_attn_prefill_f32) p_prefill_f32;
decltype(&esp_merge_partials) p_merge;
decltype(&esp_merge_partials_f32) p_merge_f32;
decltype(&esp_partial_attn_decode_shared) p_decode_shared;
decltype(&esp_qk_norm_rope_append) p_rotate;
decltype(&esp_extend_block_table) p_extend;
decltype(&esp_build_slots) p_slots;
decltype(&esp_kv_append_q4) p_append_q4;
decltype(&esp_kv_gather_q4) p_gather_q4;
decltype(&esp_partial_attn_decode_q4) p_decode_q4;
decltype(&esp_accumulate_attn_weights) p_weights;
decltype(&esp_accumulate_attn_weights_q4) p_weights_q4;
decltype(&esp_evict_slots) p_evict;

// a plain torch.Tensor (no subclass: it may answer for itself) with storage on the device
const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}
// the same, of this type, contiguous
const at::Tensor* dev(PyObject* o, at::ScalarType type) {
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}
// an output that this many elements of are written
const at::Tensor* out(PyObject* o, at::ScalarType type, int64_t numel) {
    const at::Tensor* t = dev(o, type);
    return t && t->numel() >= numel ? t : nullptr;
}
const at::Tensor* scratch(PyObject* o) {
    const at::Tensor* t = plain(o);
    return t && t->is_contiguous() ? t : nullptr;
}
bool small(PyObject* o, int32_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    v = (int32_t)x;
    return !over && x == v;
}
bool scale_of(PyObject* o, int64_t D, float& v) {
    if (o == Py_None) { v = (float)std::pow((double)D, -0.5); return D > 0; }
    if (!PyFloat_CheckExact(o)) return false;
    v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
bool fits(std::initializer_list<int64_t> sizes) {
    for (int64_t s : sizes) if (s > INT32_MAX) return false;
    return true;
}
bool stream_of(void*& s) {
    PyObject* r = PyObject_CallNoArgs(g_stream);
    if (!r) return false;
    s = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return !PyErr_Occurred();
}
// all of these (where given) on the current device
bool here(std::initializer_list<const at::Tensor*> tensors) {
    PyObject* r = PyObject_CallNoArgs(g_device);
    if (!r) return false;
    const long device = PyLong_AsLong(r);
    Py_DECREF(r);
    if (PyErr_Occurred()) return false;
    for (const at::Tensor* t : tensors) if (t && t->get_device() != device) return false;
    return true;
}
// the same for an argument that may be None: false only where it is something else that is not right
bool maybe(PyObject* o, at::ScalarType type, const at::Tensor*& t) {
    t = nullptr;
    return o == Py_None || (t = dev(o, type)) != nullptr;
}
template <class T> T* at_of(const at::Tensor* t) { return t ? (T*)t->data_ptr() : nullptr; }
// pointers of a list or tuple of tensors of one type, each of the shape `like`
struct Parts { int32_t n = 0; const void* p[ESP_MAX_PARTIALS]; };
bool parts_of(PyObject* seq, at::ScalarType type, at::IntArrayRef like, Parts& out) {
    if (!PyList_CheckExact(seq) && !PyTuple_CheckExact(seq)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    if (n > ESP_MAX_PARTIALS) return false;
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor* t = dev(PySequence_Fast_GET_ITEM(seq, i), type);
        if (!t || t->sizes() != like) return false;
        out.p[i] = t->data_ptr();
    }
    out.n = (int32_t)n;
    return true;
}

template <class F> PyObject* status_of(F call) {
    esp_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}
// a tensor may refuse to be looked at (no storage, one that stands for others): the Python meets the same and says so
template <class F> PyObject* guarded(F body) {
    PyObject* r = nullptr;
    try { r = body(); } catch (...) {}
    if (r) return r;
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

constexpr auto BF16 = at::kBFloat16;
constexpr auto F32 = at::kFloat;
constexpr auto I32 = at::kInt;

// k, v, slot_idx, k_pool, v_pool
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 5) return nullptr;
        const at::Tensor *k = dev(a[0], BF16), *v = dev(a[1], BF16), *slots = dev(a[2], I32), *kp = dev(a[3], BF16), *vp = dev(a[4], BF16);
        if (!k || !v || !slots || !kp || !vp || k->dim() != 3 || kp->dim() != 3 || slots->dim() != 1) return nullptr;
        const int64_t T = k->size(0), H = k->size(1), D = k->size(2);
        if (v->sizes() != k->sizes() || slots->size(0) != T || vp->sizes() != kp->sizes() || kp->size(1) != H || kp->size(2) != D) return nullptr;
        void* s;
        if (!fits({T, H, D}) || !stream_of(s)) return nullptr;
        const void *pk = k->data_ptr(), *pv = v->data_ptr();
        void *ppk = kp->data_ptr(), *ppv = vp->data_ptr();
        const int32_t* ps = (const int32_t*)slots->data_ptr();
        const int64_t S = kp->size(0);
        return status_of([&] { return p_append(pk, pv, ps, (int32_t)T, ppk, ppv, S, (int32_t)H, (int32_t)D, s); });
    });
}

// q, k_pool, v_pool, slot_idx, seq_offsets, max_len, softmax_scale, O, LSE, workspace[, peer_O, peer_LSE]
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 10 && n != 12) return nullptr;
        const at::Tensor *q = dev(a[0], BF16), *kp = dev(a[1], BF16), *vp = dev(a[2], BF16), *slots = dev(a[3], I32), *off = dev(a[4], I32);
        if (!q || !kp || !vp || !slots || !off || q->dim() != 3 || kp->dim() != 3) return nullptr;
        const int64_t B = q->size(0), Hq = q->size(1), D = q->size(2), S = kp->size(0), H = kp->size(1), total = slots->numel();
        const at::Tensor *O = out(a[7], BF16, q->numel()), *L = out(a[8], F32, B * Hq), *ws = scratch(a[9]);
        if (!O || !L || !ws) return nullptr;
        int32_t max_len;
        float scale;
        if (vp->sizes() != kp->sizes() || kp->size(2) != D || off->numel() != B + 1 || !small(a[5], max_len) || !scale_of(a[6], D, scale))
            return nullptr;
        Parts po, pl;
        if (n == 12 && (!parts_of(a[10], BF16, q->sizes(), po) || !parts_of(a[11], F32, q->sizes().slice(0, 2), pl) || po.n != pl.n)) return nullptr;
        void* s;
        if (!fits({B, Hq, D, H, total}) || !stream_of(s)) return nullptr;
        const void *pq = q->data_ptr(), *pk = kp->data_ptr(), *pv = vp->data_ptr();
        const int32_t *ps = (const int32_t*)slots->data_ptr(), *pf = (const int32_t*)off->data_ptr();
        void *pO = O->data_ptr(), *pw = ws->data_ptr();
        float* pL = (float*)L->data_ptr();
        const size_t wn = (size_t)ws->numel();
        return status_of([&] {
            if (n == 10)
                return p_decode(pq, pk, pv, S, ps, pf, (int32_t)B, (int32_t)total, max_len, (int32_t)Hq, (int32_t)H, (int32_t)D, scale, pO, pL, pw, wn, s);
            return p_decode_merge(pq, pk, pv, S, ps, pf, (int32_t)B, (int32_t)total, max_len, (int32_t)Hq, (int32_t)H, (int32_t)D, scale,
                                  po.p, (const float* const*)pl.p, po.n, pO, pL, pw, wn, s);
        });
    });
}

// q, k, v, q_pos, kv_pos, cu_q, cu_kv, max_q, max_kv, softmax_scale, causal, O, LSE, workspace
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 14) return nullptr;
        const at::Tensor *q = dev(a[0], BF16), *k = dev(a[1], BF16), *v = dev(a[2], BF16), *qp = dev(a[3], I32), *kp = dev(a[4], I32);
        const at::Tensor *O = plain(a[11]), *L = dev(a[12], F32), *ws = scratch(a[13]);
        if (!q || !k || !v || !qp || !kp || !O || !L || !ws || q->dim() != 3 || k->dim() != 3 || qp->dim() != 1 || kp->dim() != 1) return nullptr;
        const bool f32 = O->scalar_type() == F32;
        const int64_t Tq = q->size(0), Hq = q->size(1), D = q->size(2), Tk = k->size(0), H = k->size(1);
        if ((!f32 && O->scalar_type() != BF16) || !O->is_contiguous() || O->sizes() != q->sizes() || L->sizes() != q->sizes().slice(0, 2)) return nullptr;
        if (v->sizes() != k->sizes() || k->size(2) != D || qp->size(0) != Tq || kp->size(0) != Tk) return nullptr;
        int64_t batch = 1;
        int32_t max_q = (int32_t)Tq, max_kv = (int32_t)Tk;
        const int32_t *cq = nullptr, *ck = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor *tq = dev(a[5], I32), *tk = dev(a[6], I32);
            if (!tq || !tk || tk->numel() != tq->numel() || !small(a[7], max_q) || !small(a[8], max_kv)) return nullptr;
            batch = tq->numel() - 1;
            cq = (const int32_t*)tq->data_ptr();
            ck = (const int32_t*)tk->data_ptr();
        } else if (a[6] != Py_None) {
            return nullptr;
        }
        float scale;
        if (!scale_of(a[9], D, scale) || !PyBool_Check(a[10])) return nullptr;
        void* s;
        if (!fits({Tq, Tk, Hq, H, D, batch}) || !stream_of(s)) return nullptr;
        const int32_t causal = a[10] == Py_True ? 1 : 0;
        const void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr();
        const int32_t *pqp = (const int32_t*)qp->data_ptr(), *pkp = (const int32_t*)kp->data_ptr();
        void *pO = O->data_ptr(), *pw = ws->data_ptr();
        float* pL = (float*)L->data_ptr();
        const size_t wn = (size_t)ws->numel();
        return status_of([&] {
            if (f32)
                return p_prefill_f32(pq, pk, pv, pqp, pkp, cq, ck, (int32_t)batch, (int32_t)Tq, (int32_t)Tk, max_q, max_kv, (int32_t)Hq, (int32_t)H,
                                     (int32_t)D, scale, causal, (float*)pO, pL, pw, wn, s);
            return p_prefill(pq, pk, pv, pqp, pkp, cq, ck, (int32_t)batch, (int32_t)Tq, (int32_t)Tk, max_q, max_kv, (int32_t)Hq, (int32_t)H,
                             (int32_t)D, scale, causal, pO, pL, pw, wn, s);
        });
    });
}

// O_parts, LSE_parts, O, LSE
PyObject* merge(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 4 || (!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) || PySequence_Fast_GET_SIZE(a[0]) == 0) return nullptr;
        const at::Tensor* first = plain(PySequence_Fast_GET_ITEM(a[0], 0));
        if (!first || first->dim() < 2) return nullptr;
        const bool f32 = first->scalar_type() == F32;
        Parts po, pl;
        const auto sizes = first->sizes();
        if ((!f32 && first->scalar_type() != BF16) || !parts_of(a[0], first->scalar_type(), sizes, po) ||
            !parts_of(a[1], F32, sizes.slice(0, sizes.size() - 1), pl) || po.n != pl.n) return nullptr;
        const int64_t Hq = sizes[sizes.size() - 2], D = sizes[sizes.size() - 1];
        int64_t T = 1;
        for (size_t i = 0; i + 2 < sizes.size(); ++i) T *= sizes[i];
        const at::Tensor *O = out(a[2], BF16, first->numel()), *L = out(a[3], F32, T * Hq);
        if (!O || !L) return nullptr;
        void* s;
        if (!fits({T, Hq, D}) || !stream_of(s)) return nullptr;
        void* pO = O->data_ptr();
        float* pL = (float*)L->data_ptr();
        return status_of([&] {
            if (f32) return p_merge_f32((const float* const*)po.p, (const float* const*)pl.p, po.n, (int32_t)T, (int32_t)Hq, (int32_t)D, pO, pL, s);
            return p_merge(po.p, (const float* const*)pl.p, po.n, (int32_t)T, (int32_t)Hq, (int32_t)D, pO, pL, s);
        });
    });
}

// q, k_pool, v_pool, prefix_slots, prefix_offsets, group_offsets, max_prefix, max_group, slot_idx, seq_offsets, max_len, softmax_scale, O, LSE, workspace
PyObject* decode_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 15) return nullptr;
        const at::Tensor *q = dev(a[0], BF16), *kp = dev(a[1], BF16), *vp = dev(a[2], BF16), *ps = dev(a[3], I32), *po = dev(a[4], I32), *go = dev(a[5], I32);
        const at::Tensor *slots = dev(a[8], I32), *off = dev(a[9], I32);
        if (!q || !kp || !vp || !ps || !po || !go || !slots || !off || q->dim() != 3 || kp->dim() != 3) return nullptr;
        const int64_t B = q->size(0), Hq = q->size(1), D = q->size(2), S = kp->size(0), H = kp->size(1), groups = go->numel() - 1, P = ps->numel(), total = slots->numel();
        const at::Tensor *O = out(a[12], BF16, q->numel()), *L = out(a[13], F32, B * Hq), *ws = scratch(a[14]);
        int32_t max_prefix, max_group, max_len;
        float scale;
        if (!O || !L || !ws || vp->sizes() != kp->sizes() || kp->size(2) != D || off->numel() != B + 1 || groups < 0 || po->numel() != groups + 1 ||
            !small(a[6], max_prefix) || !small(a[7], max_group) || !small(a[10], max_len) || !scale_of(a[11], D, scale)) return nullptr;
        void* s;
        if (!fits({B, Hq, D, H, groups, P, total}) || !here({q, kp, vp, ps, po, go, slots, off, O, L, ws}) || !stream_of(s)) return nullptr;
        const size_t wn = (size_t)ws->numel() * ws->element_size();
        return status_of([&] {
            return p_decode_shared(q->data_ptr(), kp->data_ptr(), vp->data_ptr(), S, at_of<int32_t>(ps), at_of<int32_t>(po), at_of<int32_t>(go), (int32_t)groups, (int32_t)P,
                                   max_prefix, max_group, at_of<int32_t>(slots), at_of<int32_t>(off), (int32_t)B, (int32_t)total, max_len, (int32_t)Hq, (int32_t)H,
                                   (int32_t)D, scale, O->data_ptr(), at_of<float>(L), ws->data_ptr(), wn, s);
        });
    });
}

// [T, H, D] with a token's heads dense
const at::Tensor* heads(PyObject* o, int64_t& stride) {
    const at::Tensor* t = plain(o);
    if (!t || t->scalar_type() != BF16 || t->dim() != 3) return nullptr;
    const int64_t T = t->size(0), H = t->size(1), D = t->size(2);
    if ((D > 1 && t->stride(2) != 1) || (H > 1 && t->stride(1) != D)) return nullptr;
    stride = T > 1 ? t->stride(0) : H * D;
    return t;
}

// q, k, v, q_pos, inv_freq, q_weight, k_weight, eps, interleaved, slot_idx, k_pool, v_pool, q_out, k_out, v_out
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 15) return nullptr;
        int64_t qs, ks, vs, os;
        const at::Tensor *q = heads(a[0], qs), *k = heads(a[1], ks), *v = heads(a[2], vs), *qo = heads(a[12], os);
        if (!q || !k || !v || !qo) return nullptr;
        const at::Tensor *pos, *freq, *qw, *kw, *slots, *kp, *vp, *ko, *vo;
        if (!maybe(a[3], I32, pos) || !maybe(a[4], F32, freq) || !maybe(a[5], BF16, qw) || !maybe(a[6], BF16, kw) || !maybe(a[9], I32, slots) ||
            !maybe(a[10], BF16, kp) || !maybe(a[11], BF16, vp) || !maybe(a[13], BF16, ko) || !maybe(a[14], BF16, vo)) return nullptr;
        const int64_t T = q->size(0), Hq = q->size(1), D = q->size(2), H = k->size(1);
        if (k->size(0) != T || k->size(2) != D || v->sizes() != k->sizes() || qo->sizes() != q->sizes() || (freq && !pos) ||
            (pos && (pos->dim() != 1 || pos->size(0) != T)) || (qw && (qw->dim() != 1 || qw->size(0) != D)) || (kw && (kw->dim() != 1 || kw->size(0) != D)) ||
            (ko && ko->sizes() != k->sizes()) || (vo && vo->sizes() != k->sizes()) || !slots != !kp || !slots != !vp) return nullptr;
        if (slots && (slots->dim() != 1 || slots->size(0) != T || kp->dim() != 3 || kp->size(1) != H || kp->size(2) != D || vp->sizes() != kp->sizes())) return nullptr;
        if (!PyFloat_CheckExact(a[7]) || !PyBool_Check(a[8])) return nullptr;
        const int64_t rot = freq ? 2 * freq->numel() : 0;
        void* s;
        if (!fits({T, Hq, D, H, rot}) || !here({q, k, v, qo, pos, freq, qw, kw, slots, kp, vp, ko, vo}) || !stream_of(s)) return nullptr;
        const float eps = (float)PyFloat_AS_DOUBLE(a[7]);
        const int32_t neighbours = a[8] == Py_True ? 1 : 0;
        return status_of([&] {
            return p_rotate(q->data_ptr(), k->data_ptr(), v->data_ptr(), qs, ks, vs, at_of<int32_t>(pos), at_of<float>(freq), (int32_t)rot, neighbours, at_of<void>(qw),
                            at_of<void>(kw), eps, (int32_t)T, (int32_t)Hq, (int32_t)H, (int32_t)D, qo->data_ptr(), os, at_of<void>(ko), at_of<void>(vo),
                            at_of<int32_t>(slots), at_of<void>(kp), at_of<void>(vp), slots ? kp->size(0) : 0, s);
        });
    });
}

// block_table, free_pages, old_lens, new_lens, page, req_row, pages_taken
PyObject* extend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 7) return nullptr;
        const at::Tensor *table = dev(a[0], I32), *pages = dev(a[1], I32), *old = dev(a[2], I32), *now = dev(a[3], I32), *row;
        if (!table || !pages || !old || !now || !maybe(a[5], I32, row) || table->dim() != 2 || pages->dim() != 1 || old->dim() != 1) return nullptr;
        const int64_t B = old->size(0), rows = table->size(0), width = table->size(1), n_free = pages->size(0);
        const at::Tensor* taken = out(a[6], I32, B + 1);
        int32_t page;
        if (!taken || now->dim() != 1 || now->size(0) != B || !small(a[4], page) || (row ? row->dim() != 1 || row->size(0) != B : B > rows)) return nullptr;
        void* s;
        if (!fits({B, rows, width, n_free}) || !here({table, pages, old, now, row, taken}) || !stream_of(s)) return nullptr;
        return status_of([&] {
            return p_extend(at_of<int32_t>(pages), (int32_t)n_free, at_of<int32_t>(row), at_of<int32_t>(old), at_of<int32_t>(now), (int32_t)B, page, at_of<int32_t>(table),
                            (int32_t)rows, (int32_t)width, at_of<int32_t>(taken), s);
        });
    });
}

// block_table, lens, page, first_token, req_row, keep_first, keep_last, pos_first, pos_stride, capacity, seq_offsets, slot_idx, token_pos
PyObject* slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 13) return nullptr;
        const at::Tensor *table = dev(a[0], I32), *lens = dev(a[1], I32), *first, *row, *list = dev(a[11], I32), *pos;
        if (!table || !lens || !list || !maybe(a[3], I32, first) || !maybe(a[4], I32, row) || !maybe(a[12], I32, pos) || table->dim() != 2 || lens->dim() != 1) return nullptr;
        const int64_t B = lens->size(0), rows = table->size(0), width = table->size(1);
        const at::Tensor* off = out(a[10], I32, B + 1);
        int32_t page, kf, kl, pf, ps, cap = 0;
        if (!off || !small(a[2], page) || !small(a[5], kf) || !small(a[6], kl) || !small(a[7], pf) || !small(a[8], ps) || (a[9] != Py_None && !small(a[9], cap)) ||
            (first && (first->dim() != 1 || first->size(0) != B)) || (row ? row->dim() != 1 || row->size(0) != B : B > rows)) return nullptr;
        const int64_t room = a[9] == Py_None ? list->numel() : cap;
        void* s;
        if (!fits({B, rows, width, room}) || list->numel() < room || (pos && pos->numel() < room) || !here({table, lens, list, first, row, pos, off}) || !stream_of(s)) return nullptr;
        return status_of([&] {
            return p_slots(at_of<int32_t>(table), (int32_t)rows, (int32_t)width, page, at_of<int32_t>(row), at_of<int32_t>(first), at_of<int32_t>(lens), (int32_t)B, kf, kl, pf, ps,
                           (int32_t)room, at_of<int32_t>(off), at_of<int32_t>(list), at_of<int32_t>(pos), s);
        });
    });
}

// a pool in 4 bits: uint8 [S, H, 68] with a slot's heads dense
struct Q4 { int64_t S, H, slot_bytes; };
const at::Tensor* q4_pool(PyObject* o, Q4& p) {
    const at::Tensor* t = plain(o);
    if (!t || t->scalar_type() != at::kByte || t->dim() != 3 || t->size(2) != ESP_Q4_HEAD_BYTES) return nullptr;
    p.S = t->size(0);
    p.H = t->size(1);
    if (t->stride(2) != 1 || (p.H > 1 && t->stride(1) != ESP_Q4_HEAD_BYTES)) return nullptr;
    p.slot_bytes = p.S > 1 ? t->stride(0) : p.H * ESP_Q4_HEAD_BYTES;
    return t;
}
bool q4_pools(PyObject* ko, PyObject* vo, const at::Tensor*& k, const at::Tensor*& v, Q4& p) {
    Q4 other;
    k = q4_pool(ko, p);
    v = k ? q4_pool(vo, other) : nullptr;
    return v && other.S == p.S && other.H == p.H && other.slot_bytes == p.slot_bytes;
}

// k, v, slot_idx, k_pool, v_pool
PyObject* append_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 5) return nullptr;
        int64_t ks, vs;
        Q4 p;
        const at::Tensor *k = heads(a[0], ks), *v = heads(a[1], vs), *slots = dev(a[2], I32), *kp, *vp;
        if (!k || !v || !slots || !q4_pools(a[3], a[4], kp, vp, p) || v->sizes() != k->sizes() || slots->dim() != 1) return nullptr;
        const int64_t T = k->size(0), H = k->size(1), D = k->size(2);
        void* s;
        if (slots->size(0) != T || p.H != H || !fits({T, H, D}) || !here({k, v, slots, kp, vp}) || !stream_of(s)) return nullptr;
        return status_of([&] {
            return p_append_q4(k->data_ptr(), v->data_ptr(), ks, vs, at_of<int32_t>(slots), (int32_t)T, kp->data_ptr(), vp->data_ptr(), p.slot_bytes, p.S, (int32_t)H, (int32_t)D, s);
        });
    });
}

// k_pool, v_pool, slot_idx, k, v
PyObject* gather_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 5) return nullptr;
        Q4 p;
        const at::Tensor *kp, *vp, *slots = dev(a[2], I32), *k = dev(a[3], BF16), *v = dev(a[4], BF16);
        if (!slots || !k || !v || !q4_pools(a[0], a[1], kp, vp, p) || slots->dim() != 1 || k->dim() != 3 || v->sizes() != k->sizes()) return nullptr;
        const int64_t T = slots->size(0);
        void* s;
        if (k->size(0) != T || k->size(1) != p.H || k->size(2) != 128 || !fits({T, p.H}) || !here({kp, vp, slots, k, v}) || !stream_of(s)) return nullptr;
        return status_of([&] {
            return p_gather_q4(kp->data_ptr(), vp->data_ptr(), p.slot_bytes, at_of<int32_t>(slots), (int32_t)T, p.S, (int32_t)p.H, 128, k->data_ptr(), v->data_ptr(), s);
        });
    });
}

// q, k_pool, v_pool, slot_idx, seq_offsets, max_len, softmax_scale, O, LSE, workspace
PyObject* decode_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 10) return nullptr;
        Q4 p;
        const at::Tensor *q = dev(a[0], BF16), *kp, *vp, *slots = dev(a[3], I32), *off = dev(a[4], I32);
        if (!q || !slots || !off || !q4_pools(a[1], a[2], kp, vp, p) || q->dim() != 3 || slots->dim() != 1 || off->dim() != 1) return nullptr;
        const int64_t B = q->size(0), Hq = q->size(1), D = q->size(2), total = slots->numel();
        const at::Tensor *O = out(a[7], BF16, q->numel()), *L = out(a[8], F32, B * Hq), *ws = scratch(a[9]);
        int32_t max_len;
        float scale;
        if (!O || !L || !ws || off->size(0) != B + 1 || !small(a[5], max_len) || !scale_of(a[6], D, scale)) return nullptr;
        void* s;
        if (!fits({B, Hq, D, p.H, total}) || !here({q, kp, vp, slots, off, O, L, ws}) || !stream_of(s)) return nullptr;
        const size_t wn = (size_t)ws->numel() * ws->element_size();
        return status_of([&] {
            return p_decode_q4(q->data_ptr(), kp->data_ptr(), vp->data_ptr(), p.slot_bytes, p.S, at_of<int32_t>(slots), at_of<int32_t>(off), (int32_t)B, (int32_t)total, max_len,
                               (int32_t)Hq, (int32_t)p.H, (int32_t)D, scale, O->data_ptr(), at_of<float>(L), ws->data_ptr(), wn, s);
        });
    });
}

// q, LSE, k_pool, slot_idx, seq_offsets, max_len, weight_sum, q_offsets, max_q, q_pos, kv_pos, softmax_scale, decay, fresh
PyObject* weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 14) return nullptr;
        const at::Tensor *q = dev(a[0], BF16), *L = dev(a[1], F32), *kp = plain(a[2]), *slots = dev(a[3], I32), *off = dev(a[4], I32), *sums = dev(a[6], F32), *qo, *qp, *kvp;
        if (!q || !L || !kp || !slots || !off || !sums || !maybe(a[7], I32, qo) || !maybe(a[9], I32, qp) || !maybe(a[10], I32, kvp) || !qp != !kvp || q->dim() != 3 ||
            slots->dim() != 1 || off->dim() != 1 || off->size(0) < 1) return nullptr;
        const int64_t Tq = q->size(0), Hq = q->size(1), D = q->size(2), B = off->size(0) - 1, total = slots->size(0);
        const bool q4 = kp->scalar_type() == at::kByte;
        Q4 p{0, 0, 0};
        if (q4) {
            if (!q4_pool(a[2], p)) return nullptr;
        } else {
            if (!dev(a[2], BF16) || kp->dim() != 3 || kp->size(2) != D) return nullptr;
            p.S = kp->size(0);
            p.H = kp->size(1);
        }
        int32_t max_len, max_q = B > 0 ? 1 : 0, fresh;
        float scale;
        if (L->sizes() != q->sizes().slice(0, 2) || sums->dim() != 1 || sums->size(0) != p.S || !small(a[5], max_len) || !small(a[13], fresh) || !scale_of(a[11], D, scale) ||
            !PyFloat_CheckExact(a[12])) return nullptr;
        const int32_t one = max_q;                                  // query a request, without offsets
        if (a[8] != Py_None || qo)
            if (!small(a[8], max_q)) return nullptr;
        if (qo ? qo->dim() != 1 || qo->size(0) != B + 1 : max_q != one || Tq != B) return nullptr;
        if (qp && (qp->dim() != 1 || qp->size(0) != Tq || kvp->dim() != 1 || kvp->size(0) != total)) return nullptr;
        const float decay = (float)PyFloat_AS_DOUBLE(a[12]);
        void* s;
        if (!fits({Tq, Hq, D, B, p.H, total}) || !here({q, L, kp, slots, off, sums, qo, qp, kvp}) || !stream_of(s)) return nullptr;
        return status_of([&] {
            if (q4)
                return p_weights_q4(q->data_ptr(), at_of<float>(L), kp->data_ptr(), p.slot_bytes, p.S, at_of<int32_t>(slots), at_of<int32_t>(off), (int32_t)B, (int32_t)total, max_len,
                                    at_of<int32_t>(qo), (int32_t)Tq, max_q, at_of<int32_t>(qp), at_of<int32_t>(kvp), (int32_t)Hq, (int32_t)p.H, (int32_t)D, scale, decay, fresh,
                                    at_of<float>(sums), s);
            return p_weights(q->data_ptr(), at_of<float>(L), kp->data_ptr(), p.S, at_of<int32_t>(slots), at_of<int32_t>(off), (int32_t)B, (int32_t)total, max_len, at_of<int32_t>(qo),
                             (int32_t)Tq, max_q, at_of<int32_t>(qp), at_of<int32_t>(kvp), (int32_t)Hq, (int32_t)p.H, (int32_t)D, scale, decay, fresh, at_of<float>(sums), s);
        });
    });
}

// weight_sum, slot_idx, seq_offsets, max_len, budget, keep_first, keep_last, token_pos, kept_offsets, kept_slots, kept_pos, freed_offsets, freed_slots, workspace
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 14) return nullptr;
        const at::Tensor *sums = dev(a[0], F32), *slots = dev(a[1], I32), *off = dev(a[2], I32), *pos, *budgets = nullptr;
        if (!sums || !slots || !off || !maybe(a[7], I32, pos) || sums->dim() != 1 || slots->dim() != 1 || off->dim() != 1 || off->size(0) < 1) return nullptr;
        const int64_t B = off->size(0) - 1, total = slots->size(0);
        int32_t max_len, budget = 0, first, last;
        if (!PyLong_CheckExact(a[4])) {
            budgets = dev(a[4], I32);
            if (!budgets || budgets->dim() != 1 || budgets->size(0) != B) return nullptr;
        } else if (!small(a[4], budget)) {
            return nullptr;
        }
        const at::Tensor *ko = out(a[8], I32, B + 1), *ks = dev(a[9], I32), *fo = out(a[11], I32, B + 1), *fs = dev(a[12], I32), *ws = scratch(a[13]), *kp = nullptr;
        if (!ko || !ks || !fo || !fs || !ws || !small(a[3], max_len) || !small(a[5], first) || !small(a[6], last)) return nullptr;
        if (pos ? pos->dim() != 1 || pos->size(0) != total || !(kp = out(a[10], I32, ks->numel())) : a[10] != Py_None) return nullptr;
        void* s;
        if (!fits({B, total, ks->numel(), fs->numel()}) || !here({sums, slots, off, pos, budgets, ko, ks, kp, fo, fs, ws}) || !stream_of(s)) return nullptr;
        const size_t wn = (size_t)ws->numel() * ws->element_size();
        return status_of([&] {
            return p_evict(at_of<float>(sums), sums->size(0), at_of<int32_t>(slots), at_of<int32_t>(pos), at_of<int32_t>(off), (int32_t)B, (int32_t)total, max_len,
                           at_of<int32_t>(budgets), budget, first, last, (int32_t)ks->numel(), at_of<int32_t>(ko), at_of<int32_t>(ks), at_of<int32_t>(kp), (int32_t)fs->numel(),
                           at_of<int32_t>(fo), at_of<int32_t>(fs), ws->data_ptr(), wn, s);
        });
    });
}

// the functions for the stream and the device, then the addresses of the C ABI's functions in the order below
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr int N = 17;
    if (n != 2 + N) { PyErr_SetString(PyExc_TypeError, "bind: the stream and device functions and seventeen addresses"); return nullptr; }
    void* at[N];
    for (int i = 0; i < N; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i + 2]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(a[0]);
    Py_XSETREF(g_stream, a[0]);
    Py_INCREF(a[1]);
    Py_XSETREF(g_device, a[1]);
    p_append = (decltype(p_append))at[0];
    p_decode = (decltype(p_decode))at[1];
    p_decode_merge = (decltype(p_decode_merge))at[2];
    p_prefill = (decltype(p_prefill))at[3];
    p_prefill_f32 = (decltype(p_prefill_f32))at[4];
    p_merge = (decltype(p_merge))at[5];
    p_merge_f32 = (decltype(p_merge_f32))at[6];
    p_decode_shared = (decltype(p_decode_shared))at[7];
    p_rotate = (decltype(p_rotate))at[8];
    p_extend = (decltype(p_extend))at[9];
    p_slots = (decltype(p_slots))at[10];
    p_append_q4 = (decltype(p_append_q4))at[11];
    p_gather_q4 = (decltype(p_gather_q4))at[12];
    p_decode_q4 = (decltype(p_decode_q4))at[13];
    p_weights = (decltype(p_weights))at[14];
    p_weights_q4 = (decltype(p_weights_q4))at[15];
    p_evict = (decltype(p_evict))at[16];
    Py_RETURN_NONE;
}

#define ESP_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ESP_METHOD(bind), ESP_METHOD(kv_append), ESP_METHOD(decode), ESP_METHOD(prefill), ESP_METHOD(merge),
                         ESP_METHOD(decode_shared), ESP_METHOD(rotate), ESP_METHOD(extend), ESP_METHOD(slots), ESP_METHOD(append_q4), ESP_METHOD(gather_q4), ESP_METHOD(decode_q4),
                         ESP_METHOD(weights), ESP_METHOD(evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
