// The row operators' calls from Python without its per-argument cost: a small call is bound by the host (a clipped
// policy step on 24 rows runs 5.6 us on the device; marshalled in Python it takes 20 us on the host, from here 7.5; scores of
// 24 tokens with ids of 64 bits 24 and 20).
//
// Every function takes the arguments of its Python wrapper in rows.py in one fixed order, allocates the outputs
// and makes the C-ABI call of include/ears.h, if and only if everything is in its plain form already: CUDA tensors on
// the current device, of the exact type and shape, contiguous per-row arrays, ids of 32 or 64 bits.  Anything else, a refusal
// by the library included, returns None, and the wrapper goes its ordinary way, which converts, checks and raises.
// Nothing is decided here that is not decided there.
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <limits>

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/ears.h"

namespace {

struct Entry { const char* name; void* fn; };
Entry g_entries[] = {{"ears_top_logits", nullptr}, {"ears_token_logprobs", nullptr}, {"ears_token_logprobs_step", nullptr},
                     {"ears_policy_loss", nullptr}, {"ears_policy_step", nullptr}, {"ears_distill_loss", nullptr},
                     {"ears_distill_step", nullptr}, {"ears_kv_write", nullptr}, {"ears_kv_read", nullptr},
                     {"ears_kv_attention", nullptr}, {"ears_kv_attention_workspace_bytes", nullptr}};
enum { kTop, kToken, kTokenStep, kPolicyLoss, kPolicyStep, kDistillLoss, kDistillStep, kKvWrite, kKvRead, kKvAttention, kKvWorkspace };

// The arguments of one call, taken in order; `plain` falls when one is not in its plain form.
struct Args {
    PyObject* const* a;
    Py_ssize_t n, i = 0;
    bool plain = true;

    PyObject* next() {
        if (i >= n) { plain = false; return Py_None; }
        return a[i++];
    }
    // a tensor, or nullptr for None where that is allowed
    const at::Tensor* tensor(bool optional) {
        PyObject* o = next();
        if (o == Py_None) {
            if (!optional) plain = false;
            return nullptr;
        }
        if (!THPVariable_Check(o)) { plain = false; return nullptr; }
        return &THPVariable_Unpack(o);
    }
    double number() {
        PyObject* o = next();
        if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
        if (PyLong_CheckExact(o)) {
            const double v = PyLong_AsDouble(o);
            if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); plain = false; }
            return v;
        }
        plain = false;
        return 0.0;
    }
    long integer() {
        PyObject* o = next();
        if (!PyLong_CheckExact(o)) { plain = false; return 0; }
        const long v = PyLong_AsLong(o);
        if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); plain = false; }
        return v;
    }
    bool flag() { return next() == Py_True; }
    // a number, or NaN for None (a NaN that is given is not plain)
    double scale() {
        if (i < n && a[i] == Py_None) { ++i; return std::numeric_limits<double>::quiet_NaN(); }
        const double v = number();
        if (std::isnan(v)) plain = false;
        return v;
    }
};

struct Rows {
    const at::Tensor* x = nullptr;
    int dtype = 0, B = 1, R = 0, V = 0;
    int64_t sb = 0, sr = 0;
    int device = -1;
    double T = 1.0;
    const float* seq_T = nullptr;
    int32_t* status = nullptr;
    void* stream = nullptr;
    at::IntArrayRef lead;
};

bool per_row(const Rows& r, const at::Tensor* t, at::ScalarType type, at::IntArrayRef shape) {
    return t->is_cuda() && t->get_device() == r.device && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous();
}

// logits, then (after the operator's own arguments) temperature, seq_temperature, status; the current stream
bool take_logits(Args& a, Rows* r) {
    r->x = a.tensor(false);
    if (!a.plain) return false;
    const at::Tensor& x = *r->x;
    if (!x.is_cuda() || (x.dim() != 2 && x.dim() != 3) || x.numel() == 0) return false;
    switch (x.scalar_type()) {
        case at::kFloat: r->dtype = EARS_DTYPE_F32; break;
        case at::kBFloat16: r->dtype = EARS_DTYPE_BF16; break;
        case at::kHalf: r->dtype = EARS_DTYPE_F16; break;
        default: return false;
    }
    r->device = x.get_device();
    if (c10::cuda::current_device() != r->device) return false;
    const auto sizes = x.sizes(), strides = x.strides();
    const int d = (int)x.dim();
    if (strides[d - 1] != 1) return false;
    for (int i = 0; i < d; ++i)
        if (sizes[i] > INT32_MAX || strides[i] < 0) return false;
    r->V = (int)sizes[d - 1];
    r->R = (int)sizes[d - 2];
    r->sr = strides[d - 2];
    if (d == 3) { r->B = (int)sizes[0]; r->sb = strides[0]; }
    r->lead = sizes.slice(0, d - 1);
    return true;
}
bool take_rest(Args& a, Rows* r) {
    r->T = a.number();
    const at::Tensor* seq = a.tensor(true);
    const at::Tensor* status = a.tensor(true);
    if (!a.plain) return false;
    if (seq) {
        const int64_t b = r->B;
        if (!per_row(*r, seq, at::kFloat, at::IntArrayRef(&b, 1))) return false;
        r->seq_T = seq->const_data_ptr<float>();
    }
    if (status) {
        if (!status->is_cuda() || status->get_device() != r->device || status->scalar_type() != at::kInt || status->numel() != 1) return false;
        r->status = status->mutable_data_ptr<int32_t>();
    }
    r->stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)r->device).stream();
    return true;
}

const float* row_floats(const Rows& r, const at::Tensor* t, bool* plain) {
    if (!t) return nullptr;
    if (!per_row(r, t, at::kFloat, r.lead)) { *plain = false; return nullptr; }
    return t->const_data_ptr<float>();
}
// 64-bit integers, as torch's own index tensors are, count as plain too; those that 32 bits cannot hold go to the nearest that
// they can, an index of no row.  `narrow` keeps what they become.
const int32_t* ints(const Rows& r, const at::Tensor* t, at::IntArrayRef shape, at::Tensor* narrow, bool* plain) {
    if (!t) return nullptr;
    if (per_row(r, t, at::kLong, shape)) {
        *narrow = at::clamp(*t, INT32_MIN, INT32_MAX).to(at::kInt);
        t = narrow;
    }
    if (!per_row(r, t, at::kInt, shape)) { *plain = false; return nullptr; }
    return t->const_data_ptr<int32_t>();
}

at::Tensor new_out(const Rows& r, at::IntArrayRef shape, at::ScalarType type = at::kFloat) {
    return at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)r.device), std::nullopt);
}
at::Tensor row_out(const Rows& r) { return new_out(r, r.lead); }
float* data_of(const at::Tensor& t) { return t.defined() ? t.mutable_data_ptr<float>() : nullptr; }

// out_grad: None, or a tensor of the logits' shape and type
struct Grad { at::Tensor t; int64_t sb = 0, sr = 0; };
bool take_grad(const Rows& r, const at::Tensor* given, Grad* g) {
    if (!given) {
        g->t = new_out(r, r.x->sizes(), r.x->scalar_type());
    } else {
        if (!given->is_cuda() || given->get_device() != r.device || given->scalar_type() != r.x->scalar_type() ||
            given->sizes() != r.x->sizes() || given->strides().back() != 1)
            return false;
        g->t = *given;
    }
    const auto st = g->t.strides();
    g->sr = st[st.size() - 2];
    g->sb = st.size() == 3 ? st[0] : 0;
    return true;
}

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* tuple_of(std::initializer_list<at::Tensor> ts) {
    PyObject* out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = wrap(t);
        if (!o) { Py_DECREF(out); return nullptr; }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

#define EARS_ROWS(r) (r).dtype, (r).x->const_data_ptr(), (r).B, (r).R, (r).V, (r).sb, (r).sr, (r).T, (r).seq_T
#define EARS_NOT_PLAIN Py_RETURN_NONE

// C++ exceptions become the Python exceptions that torch makes of them: an allocation that fails is torch.OutOfMemoryError
template <typename F>
PyObject* guarded(F&& f) {
    HANDLE_TH_ERRORS
    return f();
    END_HANDLE_TH_ERRORS
}

// (logits, accept_len, k, T, seq_T, status)
PyObject* top_logits(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Rows r;
        if (!take_logits(a, &r)) EARS_NOT_PLAIN;
        const at::Tensor* acc = a.tensor(true);
        const long k = a.integer();
        if (!take_rest(a, &r) || k < 1 || k > EARS_MAX_TOP) EARS_NOT_PLAIN;
        const int64_t b = r.B;
        bool plain = true;
        at::Tensor narrow;
        const int32_t* lengths = ints(r, acc, at::IntArrayRef(&b, 1), &narrow, &plain);
        if (!plain) EARS_NOT_PLAIN;
        c10::SmallVector<int64_t, 4> shape(r.lead.begin(), r.lead.end());
        shape.push_back(k);
        at::Tensor values = new_out(r, shape), ids = new_out(r, shape, at::kInt), lse = row_out(r);
        const int rc = ((decltype(&ears_top_logits))g_entries[kTop].fn)(
            EARS_ROWS(r), lengths, (int)k, data_of(values), ids.mutable_data_ptr<int32_t>(),
            data_of(lse), r.status, r.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({values, ids, lse});
    });
}

// (logits, tokens, entropy, T, seq_T, status)
PyObject* token_logprobs(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Rows r;
        if (!take_logits(a, &r)) EARS_NOT_PLAIN;
        const at::Tensor* tok = a.tensor(false);
        const bool entropy = a.flag();
        if (!take_rest(a, &r)) EARS_NOT_PLAIN;
        bool plain = true;
        at::Tensor narrow;
        const int32_t* t = ints(r, tok, r.lead, &narrow, &plain);
        if (!plain) EARS_NOT_PLAIN;
        at::Tensor logp = row_out(r), H;
        if (entropy) H = row_out(r);
        const int rc = ((decltype(&ears_token_logprobs))g_entries[kToken].fn)(EARS_ROWS(r), t, data_of(logp), data_of(H), nullptr,
                                                                            r.status, r.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({logp, H});
    });
}

// (logits, tokens, d_logp, d_entropy, out_grad, T, seq_T, status)
PyObject* token_logprobs_step(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Rows r;
        if (!take_logits(a, &r)) EARS_NOT_PLAIN;
        const at::Tensor *tok = a.tensor(false), *dl = a.tensor(false), *dh = a.tensor(true), *og = a.tensor(true);
        if (!take_rest(a, &r)) EARS_NOT_PLAIN;
        bool plain = true;
        at::Tensor narrow;
        const int32_t* t = ints(r, tok, r.lead, &narrow, &plain);
        const float *l = row_floats(r, dl, &plain), *h = row_floats(r, dh, &plain);
        Grad g;
        if (!plain || !take_grad(r, og, &g)) EARS_NOT_PLAIN;
        at::Tensor logp = row_out(r), H;
        if (dh) H = row_out(r);
        const int rc = ((decltype(&ears_token_logprobs_step))g_entries[kTokenStep].fn)(
            EARS_ROWS(r), t, l, h, data_of(logp), data_of(H), g.t.mutable_data_ptr(), g.sb, g.sr, r.status, r.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({logp, H, g.t});
    });
}

// (logits, tokens, old_logp, ref_logp, advantage, clip_low, clip_high, kl_coef, entropy_coef, entropy, step, row_weight,
//  out_grad, T, seq_T, status)
PyObject* policy(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Rows r;
        if (!take_logits(a, &r)) EARS_NOT_PLAIN;
        const at::Tensor *tok = a.tensor(false), *old = a.tensor(false), *ref = a.tensor(true), *adv = a.tensor(false);
        const double lo = a.number(), hi = a.number(), kl = a.number(), ent = a.number();
        const bool entropy = a.flag(), step = a.flag();
        const at::Tensor *weight = a.tensor(true), *og = a.tensor(true);
        if (!take_rest(a, &r)) EARS_NOT_PLAIN;
        bool plain = true;
        at::Tensor narrow;
        const int32_t* t = ints(r, tok, r.lead, &narrow, &plain);
        const float *o = row_floats(r, old, &plain), *f = row_floats(r, ref, &plain), *ad = row_floats(r, adv, &plain),
                    *w = row_floats(r, weight, &plain);
        Grad g;
        if (!plain || (step && !take_grad(r, og, &g))) EARS_NOT_PLAIN;
        at::Tensor loss = row_out(r), logp = row_out(r), klt, H;
        if (ref) klt = row_out(r);
        if (entropy) H = row_out(r);
        const int rc = step ? ((decltype(&ears_policy_step))g_entries[kPolicyStep].fn)(
                                  EARS_ROWS(r), t, o, f, ad, lo, hi, kl, ent, w, data_of(loss), data_of(logp), data_of(klt), data_of(H),
                                  g.t.mutable_data_ptr(), g.sb, g.sr, r.status, r.stream)
                            : ((decltype(&ears_policy_loss))g_entries[kPolicyLoss].fn)(
                                  EARS_ROWS(r), t, o, f, ad, lo, hi, kl, ent, data_of(loss), data_of(logp), data_of(klt), data_of(H),
                                  nullptr, r.status, r.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({loss, logp, klt, H, g.t});
    });
}

// (logits, values, ids, lse, kind, mix, step, row_weight, out_grad, T, seq_T, status)
PyObject* distill(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Rows r;
        if (!take_logits(a, &r)) EARS_NOT_PLAIN;
        const at::Tensor *values = a.tensor(false), *ids = a.tensor(false), *lse = a.tensor(true);
        const long kind = a.integer();
        const double mix = a.number();
        const bool step = a.flag();
        const at::Tensor *weight = a.tensor(true), *og = a.tensor(true);
        if (!take_rest(a, &r) || ids->dim() == 0) EARS_NOT_PLAIN;
        const int64_t k = ids->sizes().back();
        if (k < 1 || k > EARS_MAX_TOP) EARS_NOT_PLAIN;
        c10::SmallVector<int64_t, 4> shape(r.lead.begin(), r.lead.end());
        shape.push_back(k);
        if (!per_row(r, values, at::kFloat, shape)) EARS_NOT_PLAIN;
        bool plain = true;
        at::Tensor narrow;
        const int32_t* id = ints(r, ids, shape, &narrow, &plain);
        const float *l = row_floats(r, lse, &plain), *w = row_floats(r, weight, &plain);
        Grad g;
        if (!plain || (step && !take_grad(r, og, &g))) EARS_NOT_PLAIN;
        at::Tensor loss = row_out(r);
        const float* v = values->const_data_ptr<float>();
        const int rc = step ? ((decltype(&ears_distill_step))g_entries[kDistillStep].fn)(EARS_ROWS(r), (int)k, v, id, l, (int)kind, mix, w,
                                                                                       data_of(loss), g.t.mutable_data_ptr(), g.sb,
                                                                                       g.sr, r.status, r.stream)
                            : ((decltype(&ears_distill_loss))g_entries[kDistillLoss].fn)(EARS_ROWS(r), (int)k, v, id, l, (int)kind, mix,
                                                                                       data_of(loss), nullptr, r.status, r.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({loss, g.t});
    });
}

// ---- the key/value cache ----
struct Kv {
    ears_kv_cache cache = {};
    int device = -1, B = 0, width = 0;
    int64_t stride = 0;
    const int32_t *table = nullptr, *start = nullptr, *counts = nullptr;
    int32_t* status = nullptr;
    void* stream = nullptr;
};
bool on(const at::Tensor* t, int device, at::ScalarType type) { return t->is_cuda() && t->get_device() == device && t->scalar_type() == type; }

bool take_cache(Args& a, Kv* kv) {
    const at::Tensor *codes = a.tensor(false), *params = a.tensor(false);
    if (!a.plain || !codes->is_cuda() || codes->dim() != 5 || params->dim() != 6) return false;
    if (params->requires_grad() && c10::GradMode::is_enabled()) return false;        // refused by the wrapper
    kv->device = codes->get_device();
    if (c10::cuda::current_device() != kv->device) return false;
    if (codes->scalar_type() != at::kByte || !on(params, kv->device, at::kBFloat16) || !codes->is_contiguous() || !params->is_contiguous()) return false;
    const auto c = codes->sizes(), p = params->sizes();
    if (c[1] != 2 || c[4] > 128 || p[4] != c[4] * 2 / EARS_KV_GROUP || p[5] != 2 || c.slice(0, 4) != p.slice(0, 4)) return false;
    for (int i = 0; i < 5; ++i)
        if (c[i] > INT32_MAX) return false;
    kv->cache = {codes->mutable_data_ptr(), params->mutable_data_ptr(), (int)c[0], (int)c[2], (int)c[3], (int)c[4] * 2};
    return true;
}
bool take_seqs(Kv* kv, const at::Tensor* pages, const at::Tensor* start, const at::Tensor* counts, const at::Tensor* status) {
    if (!on(pages, kv->device, at::kInt) || pages->dim() != 2 || pages->size(0) > INT32_MAX || pages->size(1) > INT32_MAX) return false;
    if (pages->size(1) > 1 && pages->stride(1) != 1) return false;
    kv->B = (int)pages->size(0);
    kv->width = (int)pages->size(1);
    kv->stride = pages->stride(0);
    kv->table = pages->const_data_ptr<int32_t>();
    const int64_t b = kv->B;
    for (const at::Tensor* t : {start, counts})
        if (t && (!on(t, kv->device, at::kInt) || t->sizes() != at::IntArrayRef(&b, 1) || !t->is_contiguous())) return false;
    kv->start = start->const_data_ptr<int32_t>();
    kv->counts = counts ? counts->const_data_ptr<int32_t>() : nullptr;
    if (status) {
        if (!on(status, kv->device, at::kInt) || status->numel() != 1) return false;
        kv->status = status->mutable_data_ptr<int32_t>();
    }
    kv->stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)kv->device).stream();
    return true;
}
int dtype_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return EARS_DTYPE_F32;
        case at::kBFloat16: return EARS_DTYPE_BF16;
        case at::kHalf: return EARS_DTYPE_F16;
        default: return -1;
    }
}
// [B, Q, heads, head_dim], used where it lies
bool heads_of(const Kv& kv, const at::Tensor* t) {
    if (!t->is_cuda() || t->get_device() != kv.device || t->dim() != 4 || t->size(0) != kv.B || t->size(3) != kv.cache.head_dim) return false;
    if (t->requires_grad() && c10::GradMode::is_enabled()) return false;      // refused by the wrapper
    if (t->stride(3) != 1 || t->numel() == 0 || t->size(1) > INT32_MAX || t->size(2) > INT32_MAX) return false;
    return t->stride(0) >= 0 && t->stride(1) >= 0 && t->stride(2) >= 0;
}
at::Tensor kv_out(const Kv& kv, at::IntArrayRef shape, at::ScalarType type) {
    return at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)kv.device), std::nullopt);
}
#define EARS_SEQS(kv) (kv).table, (kv).width, (kv).stride, (kv).start, (kv).counts

// (codes, params, k, v, pages, start, counts, status) -> True
PyObject* kv_write(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Kv kv;
        if (!take_cache(a, &kv)) EARS_NOT_PLAIN;
        const at::Tensor *k = a.tensor(false), *v = a.tensor(false), *pages = a.tensor(false), *start = a.tensor(false), *counts = a.tensor(true),
                         *status = a.tensor(true);
        if (!a.plain || !take_seqs(&kv, pages, start, counts, status) || !heads_of(kv, k) || !heads_of(kv, v)) EARS_NOT_PLAIN;
        const int dtype = dtype_of(*k);
        if (dtype < 0 || dtype_of(*v) != dtype || k->sizes() != v->sizes() || k->size(2) != kv.cache.heads) EARS_NOT_PLAIN;
        const int rc = ((decltype(&ears_kv_write))g_entries[kKvWrite].fn)(
            dtype, &kv.cache, k->const_data_ptr(), v->const_data_ptr(), kv.B, (int)k->size(1), k->stride(0), k->stride(1), k->stride(2),
            v->stride(0), v->stride(1), v->stride(2), EARS_SEQS(kv), kv.status, kv.stream);
        if (rc) EARS_NOT_PLAIN;
        Py_RETURN_TRUE;
    });
}

// (codes, params, pages, start, tokens, counts, dtype, status)
PyObject* kv_read(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Kv kv;
        if (!take_cache(a, &kv)) EARS_NOT_PLAIN;
        const at::Tensor *pages = a.tensor(false), *start = a.tensor(false);
        const long tokens = a.integer();
        const at::Tensor* counts = a.tensor(true);
        const long dtype = a.integer();
        const at::Tensor* status = a.tensor(true);
        if (!a.plain || !take_seqs(&kv, pages, start, counts, status) || kv.B < 1 || tokens < 1 || tokens > INT32_MAX) EARS_NOT_PLAIN;
        if (dtype != EARS_DTYPE_F32 && dtype != EARS_DTYPE_BF16 && dtype != EARS_DTYPE_F16) EARS_NOT_PLAIN;
        const at::ScalarType type = dtype == EARS_DTYPE_F32 ? at::kFloat : dtype == EARS_DTYPE_BF16 ? at::kBFloat16 : at::kHalf;
        const int64_t shape[4] = {kv.B, tokens, kv.cache.heads, kv.cache.head_dim};
        at::Tensor k = kv_out(kv, shape, type), v = kv_out(kv, shape, type);
        const int rc = ((decltype(&ears_kv_read))g_entries[kKvRead].fn)((int)dtype, &kv.cache, kv.B, (int)tokens, EARS_SEQS(kv),
                                                                        k.mutable_data_ptr(), v.mutable_data_ptr(), kv.status, kv.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({k, v});
    });
}

// (codes, params, q, pages, start, counts, scale, window, sinks, lse, status)
PyObject* kv_attention(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Args a{argv, n};
        Kv kv;
        if (!take_cache(a, &kv)) EARS_NOT_PLAIN;
        const at::Tensor *q = a.tensor(false), *pages = a.tensor(false), *start = a.tensor(false), *counts = a.tensor(true);
        const double given = a.scale();
        const long window = a.integer(), sinks = a.integer();
        const bool lse = a.flag();
        const at::Tensor* status = a.tensor(true);
        if (!a.plain || !take_seqs(&kv, pages, start, counts, status) || !heads_of(kv, q)) EARS_NOT_PLAIN;
        const int dtype = dtype_of(*q), Q = (int)q->size(1), heads = (int)q->size(2);
        if ((dtype != EARS_DTYPE_BF16 && dtype != EARS_DTYPE_F16) || window < 0 || window > INT32_MAX || sinks < 0 || sinks > INT32_MAX) EARS_NOT_PLAIN;
        const double scale = std::isnan(given) ? 1.0 / std::sqrt((double)kv.cache.head_dim) : given;
        const size_t need = ((decltype(&ears_kv_attention_workspace_bytes))g_entries[kKvWorkspace].fn)(dtype, &kv.cache, kv.B, Q, heads, kv.width,
                                                                                                   (int)window, (int)sinks);
        if (!need) EARS_NOT_PLAIN;
        const int64_t bytes = (int64_t)need;
        at::Tensor out = kv_out(kv, q->sizes(), q->scalar_type()), work = kv_out(kv, at::IntArrayRef(&bytes, 1), at::kByte), sums;
        if (lse) sums = kv_out(kv, q->sizes().slice(0, 3), at::kFloat);
        const int rc = ((decltype(&ears_kv_attention))g_entries[kKvAttention].fn)(
            dtype, &kv.cache, q->const_data_ptr(), kv.B, Q, heads, q->stride(0), q->stride(1), q->stride(2), EARS_SEQS(kv), scale, (int)window,
            (int)sinks, out.mutable_data_ptr(), lse ? sums.mutable_data_ptr<float>() : nullptr, work.mutable_data_ptr(), need, kv.status, kv.stream);
        if (rc) EARS_NOT_PLAIN;
        return tuple_of({out, sums});
    });
}

// bind({name: address}): the entry points of the library in use
PyObject* bind(PyObject*, PyObject* dict) {
    for (Entry& e : g_entries) {
        PyObject* v = PyDict_Check(dict) ? PyDict_GetItemString(dict, e.name) : nullptr;
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (!p) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_KeyError, "%s", e.name);
            return nullptr;
        }
        e.fn = p;
    }
    Py_RETURN_NONE;
}

#define EARS_METHOD(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {EARS_METHOD("top_logits", top_logits), EARS_METHOD("token_logprobs", token_logprobs),
                           EARS_METHOD("token_logprobs_step", token_logprobs_step), EARS_METHOD("policy", policy),
                           EARS_METHOD("distill", distill), EARS_METHOD("kv_write", kv_write), EARS_METHOD("kv_read", kv_read),
                           EARS_METHOD("kv_attention", kv_attention), {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "ears_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_ears_torch(void) {
    PyObject* m = PyModule_Create(&g_module);
    // what build.py compares before it takes a module that is there already, and the C interface's version
    if (m && (PyModule_AddStringConstant(m, "stamp", EARS_TORCH_STAMP) || PyModule_AddIntConstant(m, "version", EARS_VERSION))) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
