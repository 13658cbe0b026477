// The calls of mcf_cache.h on torch tensors.  A CPython extension as mcf_torch.cpp is, for the same reason.
#include "torch_call.h"

#include <ATen/core/grad_mode.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/mcf_cache.h"

namespace mcf {
int check_norm_rotate(const mcf_norm_rotate_call *c, bool back); // all that a call is checked for, on the host
int check_append(const mcf_append_call *c);
int check_attention(const mcf_attention_call *c);
} // namespace mcf

namespace {

struct Refused { // an error to raise, on the way out of nested checks
    int status;
    const char *text;
};

const at::Tensor *tensor(PyObject *o, const char *missing) { // missing: what to say of None, nullptr where that is fine
    if (o == Py_None) {
        if (missing) throw Refused{MCF_EINVAL, missing};
        return nullptr;
    }
    if (!THPVariable_Check(o)) throw Refused{MCF_EINVAL, "tensors are expected"};
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided) throw Refused{MCF_EUNSUPPORTED, "tensors are strided"};
    return &t;
}

// What the tensors of a call have in common: the device, checked after everything else.
struct Operands {
    const at::Tensor *all[24];
    int n = 0;
    void add(const at::Tensor *t) {
        if (t) all[n++] = t;
    }
    c10::Device device() const {
        for (int i = 0; i < n; ++i) {
            if (!all[i]->is_cuda()) throw Refused{MCF_EINVAL, "operands must be device tensors"};
            if (all[i]->device() != all[0]->device()) throw Refused{MCF_EINVAL, "operands must live on one device"};
        }
        return all[0]->device();
    }
};

// [batch, tokens, heads, size] or [tokens, heads, size], last dimension packed
mcf_rows rows(const at::Tensor &t) {
    mcf_rows r;
    const int64_t d = t.dim();
    if (d != 3 && d != 4) throw Refused{MCF_EINVAL, "rows are [tokens, heads, size] or [batch, tokens, heads, size]"};
    if (t.size(d - 1) > 1 && t.stride(d - 1) != 1) throw Refused{MCF_EUNSUPPORTED, "the last dimension of rows is packed"};
    r.data = t.data_ptr();
    r.stride[0] = d == 4 ? t.stride(0) : 0;
    r.stride[1] = t.stride(d - 3);
    r.stride[2] = t.stride(d - 2);
    return r;
}
int dtype_of(const at::Tensor &t) {
    if (t.scalar_type() == at::kHalf) return MCF_F16;
    if (t.scalar_type() == at::kBFloat16) return MCF_BF16;
    throw Refused{MCF_EUNSUPPORTED, "rows are float16 or bfloat16"};
}
void same(const at::Tensor &a, const at::Tensor &b, const char *text) {
    if (a.scalar_type() != b.scalar_type() || a.sizes() != b.sizes()) throw Refused{MCF_EINVAL, text};
}

void tables(const at::Tensor *cos, const at::Tensor *sin, const float **c, const float **s, int64_t *rotary, int64_t *rows) {
    *c = *s = nullptr;
    *rotary = *rows = 0;
    if (!cos && !sin) return;
    if (!cos || !sin) throw Refused{MCF_EINVAL, "cos and sin come together"};
    for (const at::Tensor *t : {cos, sin})
        if (t->dim() != 2 || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->sizes() != cos->sizes())
            throw Refused{MCF_EINVAL, "cos and sin are packed float32 [positions, rotary / 2]"};
    *c = (const float *)cos->data_ptr();
    *s = (const float *)sin->data_ptr();
    *rotary = 2 * cos->size(1);
    *rows = cos->size(0);
}

const void *weight(const at::Tensor *w, int64_t size, const at::Tensor &x, int *f32) { // *f32: -1 before the first weight
    if (!w) return nullptr;
    if (w->dim() != 1 || w->size(0) != size || (size > 1 && w->stride(0) != 1)) throw Refused{MCF_EINVAL, "a weight is packed [size]"};
    const bool is_f32 = w->scalar_type() == at::kFloat;
    if (!is_f32 && w->scalar_type() != x.scalar_type()) throw Refused{MCF_EINVAL, "weights have the type of the rows, or float32"};
    if (*f32 >= 0 && *f32 != (int)is_f32) throw Refused{MCF_EINVAL, "both weights have one type"};
    *f32 = is_f32;
    return w->data_ptr();
}

double number(PyObject *o) {
    PyObject *f = PyNumber_Float(o);
    if (!f) return 0.0;
    const double x = PyFloat_AsDouble(f);
    Py_DECREF(f);
    return x;
}

void *stream_of(PyObject *o, c10::Device device) {
    return o == Py_None ? (void *)c10::hip::getCurrentHIPStream(device.index()).stream() : PyLong_AsVoidPtr(o);
}

// The device and the stream of a call.  Where that is not torch's current stream, what the call makes is memory of its stream, and neither
// that nor what the caller brought is handed out again before both streams are through with it.  (While the stream is captured, by whomever, no events
// may be recorded on it: memory that a graph uses is its owner's to keep.)
struct Place {
    const c10::DeviceGuard on;
    const c10::hip::HIPStream here, there;
    const bool other;
    Place(c10::Device device, void *stream)
        : on(device), here(c10::hip::getCurrentHIPStream(device.index())),
          there(here.stream() == (hipStream_t)stream ? here : c10::hip::getStreamFromExternal((hipStream_t)stream, device.index())),
          other(here.stream() != there.stream() && !mcf::stream_capturing(there.stream())) {
        if (other) c10::hip::setCurrentHIPStream(there);
    }
    ~Place() {
        if (other) c10::hip::setCurrentHIPStream(here);
    }
    Place(const Place &) = delete;
    void used(const Operands &brought, std::initializer_list<const at::Tensor *> made) const { // after the launches
        if (!other) return;
        for (int i = 0; i < brought.n; ++i) c10::hip::HIPCachingAllocator::recordStream(brought.all[i]->storage().data_ptr(), there);
        for (const at::Tensor *t : made)
            if (t->defined()) c10::hip::HIPCachingAllocator::recordStream(t->storage().data_ptr(), here);
    }
};

void status(int st) {
    if (st == MCF_OK) return;
    static thread_local char text[512];
    const char *more = mcf_last_error();
    snprintf(text, sizeof(text), *more ? "%s (%s)" : "%s", mcf_status_string(st), more);
    throw Refused{st, text};
}

PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }

// The results of rows x where the caller gives none.
at::Tensor like(const at::Tensor &x) { return at::empty(x.sizes(), x.options()); }

// q, k and their common arguments of both norm_rotate calls
void norm_rotate_operands(mcf_norm_rotate_call &c, Operands &ops, const at::Tensor *q, const at::Tensor *k, PyObject *const *arg, PyObject *eps, PyObject *interleaved) {
    const at::Tensor *cos = tensor(arg[0], nullptr), *sin = tensor(arg[1], nullptr), *positions = tensor(arg[2], nullptr), *qw = tensor(arg[3], nullptr),
                     *kw = tensor(arg[4], nullptr);
    for (const at::Tensor *t : {q, k, cos, sin, positions, qw, kw}) ops.add(t);
    memset(&c, 0, sizeof(c));
    c.dtype = dtype_of(*q);
    c.q = rows(*q);
    const int64_t d = q->dim();
    c.batch = d == 4 ? q->size(0) : 1;
    c.tokens = q->size(d - 3); c.q_heads = q->size(d - 2); c.size = q->size(d - 1);
    if (k) {
        c.k = rows(*k);
        if (k->dim() != d || k->scalar_type() != q->scalar_type() || k->size(d - 1) != c.size || k->size(d - 3) != c.tokens || (d == 4 && k->size(0) != c.batch))
            throw Refused{MCF_EINVAL, "q and k differ in type, tokens or size"};
        c.k_heads = k->size(d - 2);
    }
    tables(cos, sin, &c.cos, &c.sin, &c.rotary, &c.table_rows);
    int f32 = -1;
    c.q_weight = weight(qw, c.size, *q, &f32);
    c.k_weight = weight(k ? kw : nullptr, c.size, *q, &f32);
    c.weight_f32 = f32 > 0;
    if (positions) {
        if (positions->scalar_type() != at::kInt && positions->scalar_type() != at::kLong) throw Refused{MCF_EINVAL, "positions are int32 or int64"};
        const bool each = d == 4 && positions->dim() == 2;
        if (!positions->is_contiguous() || (each ? positions->size(0) != c.batch : positions->dim() != 1) || positions->size(-1) != c.tokens)
            throw Refused{MCF_EINVAL, "positions are packed, one for each token"};
        c.positions = positions->data_ptr();
        c.position_bytes = positions->scalar_type() == at::kInt ? 4 : 8;
        c.position_batch = each ? c.tokens : 0;
    }
    c.eps = number(eps);
    c.interleaved = PyObject_IsTrue(interleaved);
    if (PyErr_Occurred()) throw Refused{0, nullptr};
}

// Whether a call is to be recorded for autograd, which Python does (NotImplemented): into new tensors, outside of captures.
bool recorded(std::initializer_list<const at::Tensor *> operands, std::initializer_list<const at::Tensor *> tables, bool results_given) {
    const auto wanted = [](const at::Tensor *t) { return t && t->requires_grad(); };
    if (!at::GradMode::is_enabled()) return false;
    if (std::any_of(tables.begin(), tables.end(), wanted)) throw Refused{MCF_EUNSUPPORTED, "the tables have no gradients"};
    if (std::none_of(operands.begin(), operands.end(), wanted)) return false;
    if (results_given) throw Refused{MCF_EUNSUPPORTED, "results in tensors of the caller are not recorded for autograd (torch.no_grad() and norm_rotate_backward)"};
    return true;
}

// norm_rotate(q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, q_out, k_out, stream) -> (q_out, k_out), or NotImplemented: to be recorded
PyObject *norm_rotate(PyObject *const *arg, Py_ssize_t n) {
    if (n != 12) return PyErr_Format(PyExc_TypeError, "norm_rotate takes 12 arguments");
    const at::Tensor *q = tensor(arg[0], "q is missing"), *k = tensor(arg[1], nullptr), *qo = tensor(arg[9], nullptr), *ko = tensor(arg[10], nullptr);
    mcf_norm_rotate_call c;
    Operands ops;
    norm_rotate_operands(c, ops, q, k, arg + 2, arg[7], arg[8]);
    ops.add(qo);
    if (ko && !k) throw Refused{MCF_EINVAL, "k_out without k"};
    ops.add(ko);
    at::Tensor qn, kn;
    if (qo) same(*qo, *q, "q_out has another shape or type than q");
    if (ko) same(*ko, *k, "k_out has another shape or type than k");
    mcf_rows packed_q = {q->data_ptr(), {c.tokens * c.q_heads * c.size, c.q_heads * c.size, c.size}};
    c.q_out = qo ? rows(*qo) : packed_q;
    if (k) c.k_out = ko ? rows(*ko) : mcf_rows{k->data_ptr(), {c.tokens * c.k_heads * c.size, c.k_heads * c.size, c.size}};
    status(mcf::check_norm_rotate(&c, false));
    const bool record = recorded({q, k, tensor(arg[5], nullptr), tensor(arg[6], nullptr)}, {tensor(arg[2], nullptr), tensor(arg[3], nullptr)}, qo || ko);
    const c10::Device device = ops.device();
    void *stream = stream_of(arg[11], device);
    if (PyErr_Occurred()) return nullptr;
    if (record) {
        if (mcf::stream_capturing(stream))
            throw Refused{MCF_EUNSUPPORTED, "a call that is captured is not recorded for autograd (torch.no_grad() and norm_rotate_backward)"};
        return Py_NewRef(Py_NotImplemented);
    }
    int st;
    {
        const NoGil released;
        const Place place(device, stream);
        if (!qo) { qn = like(*q); c.q_out = rows(qn); }
        if (k && !ko) { kn = like(*k); c.k_out = rows(kn); }
        st = mcf_norm_rotate(&c, stream);
        place.used(ops, {&qn, &kn});
    }
    status(st);
    return Py_BuildValue("(NN)", wrap(qo ? *qo : qn), k ? wrap(ko ? *ko : kn) : Py_NewRef(Py_None));
}

// norm_rotate_backward(dq, dk, q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, q_out, k_out, stream)
//   -> (gradient of q, of k, of q_weight, of k_weight), None for what is not there
PyObject *norm_rotate_backward(PyObject *const *arg, Py_ssize_t n) {
    if (n != 14) return PyErr_Format(PyExc_TypeError, "norm_rotate_backward takes 14 arguments");
    const at::Tensor *dq = tensor(arg[0], "dq is missing"), *dk = tensor(arg[1], nullptr), *q = tensor(arg[2], "q is missing"), *k = tensor(arg[3], nullptr),
                     *qo = tensor(arg[11], nullptr), *ko = tensor(arg[12], nullptr);
    mcf_norm_rotate_call c;
    Operands ops;
    norm_rotate_operands(c, ops, q, k, arg + 4, arg[9], arg[10]);
    for (const at::Tensor *t : {dq, dk, qo, ko}) ops.add(t);
    if (!k != !dk || (ko && !k)) throw Refused{MCF_EINVAL, "k and its gradients come together"};
    same(*dq, *q, "dq has another shape or type than q");
    if (k) same(*dk, *k, "dk has another shape or type than k");
    if (qo) same(*qo, *q, "q_out has another shape or type than q");
    if (ko) same(*ko, *k, "k_out has another shape or type than k");
    c.dq = rows(*dq);
    if (k) c.dk = rows(*dk);
    c.q_out = qo ? rows(*qo) : mcf_rows{q->data_ptr(), {c.tokens * c.q_heads * c.size, c.q_heads * c.size, c.size}};
    if (k) c.k_out = ko ? rows(*ko) : mcf_rows{k->data_ptr(), {c.tokens * c.k_heads * c.size, c.k_heads * c.size, c.size}};
    float stand_in;
    c.dq_weight = c.dk_weight = &stand_in;
    status(mcf::check_norm_rotate(&c, true));
    const c10::Device device = ops.device();
    void *stream = stream_of(arg[13], device);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor qn, kn, qw, kw;
    int st;
    {
        const NoGil released;
        const Place place(device, stream);
        if (!qo) { qn = like(*q); c.q_out = rows(qn); }
        if (k && !ko) { kn = like(*k); c.k_out = rows(kn); }
        const at::TensorOptions f32 = q->options().dtype(at::kFloat);
        c.dq_weight = c.dk_weight = nullptr;
        if (c.q_weight) { qw = at::empty({c.size}, f32); c.dq_weight = (float *)qw.data_ptr(); }
        if (c.k_weight) { kw = at::empty({c.size}, f32); c.dk_weight = (float *)kw.data_ptr(); }
        int64_t bytes = 0;
        st = mcf_norm_rotate_backward_workspace(&c, &bytes);
        void *ws = nullptr;
        if (st == MCF_OK && bytes > 0) {
            ws = workspace((size_t)bytes, (hipStream_t)stream, device);
            if (!ws) {
                mcf::set_last_error("gradients of weights in a graph that torch does not capture");
                st = MCF_EUNSUPPORTED;
            }
        }
        if (st == MCF_OK) st = mcf_norm_rotate_backward(&c, ws, bytes, stream);
        if (ws) c10::hip::HIPCachingAllocator::raw_delete(ws);
        place.used(ops, {&qn, &kn, &qw, &kw});
    }
    status(st);
    const auto or_none = [](const at::Tensor &t) { return t.defined() ? wrap(t) : Py_NewRef(Py_None); };
    return Py_BuildValue("(NNNN)", wrap(qo ? *qo : qn), ko ? wrap(*ko) : or_none(kn), or_none(qw), or_none(kw));
}

// cache: the tuple (k, v, k_scale, v_scale)
mcf_kv_cache cache_of(PyObject *o, Operands &ops) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) throw Refused{MCF_EINVAL, "a cache is a KVCache"};
    const at::Tensor *t[4];
    for (int i = 0; i < 4; ++i) {
        t[i] = tensor(PyTuple_GET_ITEM(o, i), "a part of the cache is missing");
        ops.add(t[i]);
    }
    mcf_kv_cache c;
    for (int i = 0; i < 2; ++i) {
        if (t[i]->dim() != 4 || t[i]->scalar_type() != at::kFloat8_e4m3fn || t[i]->sizes() != t[0]->sizes())
            throw Refused{MCF_EINVAL, "the pages are float8_e4m3fn [pages, heads, page_size, size]"};
        if ((t[i]->size(3) > 1 && t[i]->stride(3) != 1) || (t[i]->size(2) > 1 && t[i]->stride(2) != t[i]->size(3)))
            throw Refused{MCF_EUNSUPPORTED, "the tokens of a page and head are packed"};
        if (t[2 + i]->dim() != 2 || t[2 + i]->scalar_type() != at::kFloat || t[2 + i]->size(0) != t[0]->size(0) || t[2 + i]->size(1) != t[0]->size(1))
            throw Refused{MCF_EINVAL, "the scales are float32 [pages, heads]"};
        if (t[2 + i]->size(1) > 1 && t[2 + i]->stride(1) != 1) throw Refused{MCF_EUNSUPPORTED, "the scales of a page are packed"};
    }
    c.pages = t[0]->size(0); c.heads = t[0]->size(1); c.page_size = t[0]->size(2); c.size = t[0]->size(3);
    c.k = t[0]->data_ptr(); c.v = t[1]->data_ptr();
    c.k_scale = (float *)t[2]->data_ptr(); c.v_scale = (float *)t[3]->data_ptr();
    c.k_stride[0] = t[0]->stride(0); c.k_stride[1] = t[0]->stride(1);
    c.v_stride[0] = t[1]->stride(0); c.v_stride[1] = t[1]->stride(1);
    c.k_scale_stride = t[2]->stride(0); c.v_scale_stride = t[3]->stride(0);
    return c;
}

mcf_sequences sequences_of(PyObject *table, PyObject *lengths, PyObject *starts, int64_t tokens, Operands &ops) {
    const at::Tensor *t = tensor(table, "the table is missing"), *l = tensor(lengths, "the lengths are missing"), *s = tensor(starts, nullptr);
    for (const at::Tensor *x : {t, l, s}) {
        ops.add(x);
        if (x && x->scalar_type() != at::kInt) throw Refused{MCF_EINVAL, "table, lengths and starts are int32"};
    }
    if (t->dim() != 2 || l->dim() != 1 || t->size(0) != l->size(0)) throw Refused{MCF_EINVAL, "the table is [sequences, pages], the lengths [sequences]"};
    if (s && (s->dim() != 1 || s->size(0) != l->size(0) + 1)) throw Refused{MCF_EINVAL, "starts has one entry more than there are sequences"};
    if ((t->size(1) > 1 && t->stride(1) != 1) || (l->size(0) > 1 && l->stride(0) != 1) || (s && s->size(0) > 1 && s->stride(0) != 1))
        throw Refused{MCF_EUNSUPPORTED, "rows of the table, lengths and starts are packed"};
    if (!s && l->size(0) != tokens) throw Refused{MCF_EINVAL, "without starts every sequence has one row"};
    mcf_sequences q;
    q.batch = l->size(0); q.tokens = tokens;
    q.table_width = t->size(1); q.table_stride = t->stride(0);
    q.starts = s ? (const int32_t *)s->data_ptr() : nullptr;
    q.lengths = (const int32_t *)l->data_ptr();
    q.table = (const int32_t *)t->data_ptr();
    return q;
}

const at::Tensor &three(const at::Tensor *t) {
    if (t->dim() != 3) throw Refused{MCF_EINVAL, "rows are [tokens, heads, size]"};
    return *t;
}

// append_cache(cache, k, v, table, lengths, starts, cos, sin, k_weight, q, q_weight, eps, interleaved, q_out, stream) -> q_out
PyObject *append_cache(PyObject *const *arg, Py_ssize_t n) {
    if (n != 15) return PyErr_Format(PyExc_TypeError, "append_cache takes 15 arguments");
    Operands ops;
    mcf_append_call c;
    memset(&c, 0, sizeof(c));
    c.cache = cache_of(arg[0], ops);
    const at::Tensor *k = tensor(arg[1], "k is missing"), *v = tensor(arg[2], "v is missing"), *q = tensor(arg[9], nullptr), *qo = tensor(arg[13], nullptr);
    const at::Tensor *cos = tensor(arg[6], nullptr), *sin = tensor(arg[7], nullptr), *kw = tensor(arg[8], nullptr), *qw = tensor(arg[10], nullptr);
    for (const at::Tensor *t : {k, v, q, qo, cos, sin, kw, qw}) ops.add(t);
    c.dtype = dtype_of(*k);
    c.k = rows(three(k)); c.v = rows(three(v));
    same(*k, *v, "k and v differ in shape or type");
    if (k->size(1) != c.cache.heads || k->size(2) != c.cache.size) throw Refused{MCF_EINVAL, "k and v have other heads or another size than the cache"};
    c.seq = sequences_of(arg[3], arg[4], arg[5], k->size(0), ops);
    tables(cos, sin, &c.cos, &c.sin, &c.rotary, &c.table_rows);
    int f32 = -1;
    c.k_weight = weight(kw, c.cache.size, *k, &f32);
    if (q) {
        c.q = rows(three(q));
        if (q->scalar_type() != k->scalar_type() || q->size(0) != k->size(0) || q->size(2) != k->size(2)) throw Refused{MCF_EINVAL, "q and k differ in type, tokens or size"};
        c.q_heads = q->size(1);
        c.q_weight = weight(qw, c.cache.size, *q, &f32);
        if (qo) same(*qo, *q, "q_out has another shape or type than q");
        c.q_out = qo ? rows(*qo) : mcf_rows{q->data_ptr(), {0, c.q_heads * c.cache.size, c.cache.size}};
    } else if (qo || qw) {
        throw Refused{MCF_EINVAL, "q_out or q_weight without q"};
    }
    c.weight_f32 = f32 > 0;
    c.eps = number(arg[11]);
    c.interleaved = PyObject_IsTrue(arg[12]);
    if (PyErr_Occurred()) return nullptr;
    status(mcf::check_append(&c));
    const c10::Device device = ops.device();
    void *stream = stream_of(arg[14], device);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor qn;
    int st;
    {
        const NoGil released;
        const Place place(device, stream);
        if (q && !qo) { qn = like(*q); c.q_out = rows(qn); }
        st = mcf_cache_append(&c, stream);
        place.used(ops, {&qn});
    }
    status(st);
    return q ? wrap(qo ? *qo : qn) : Py_NewRef(Py_None);
}

// cache_attention(q, cache, table, lengths, scale, starts, causal, out, stream) -> out
PyObject *cache_attention(PyObject *const *arg, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "cache_attention takes 9 arguments");
    Operands ops;
    mcf_attention_call c;
    memset(&c, 0, sizeof(c));
    const at::Tensor *q = tensor(arg[0], "q is missing"), *out = tensor(arg[7], nullptr);
    ops.add(q);
    ops.add(out);
    c.cache = cache_of(arg[1], ops);
    c.dtype = dtype_of(*q);
    c.q = rows(three(q));
    if (q->size(2) != c.cache.size) throw Refused{MCF_EINVAL, "q has another size than the cache"};
    c.q_heads = q->size(1);
    c.seq = sequences_of(arg[2], arg[3], arg[5], q->size(0), ops);
    if (out) same(*out, *q, "out has another shape or type than q");
    c.out = out ? rows(*out) : mcf_rows{q->data_ptr(), {0, c.q_heads * c.cache.size, c.cache.size}};
    c.scale = (float)number(arg[4]);
    c.causal = PyObject_IsTrue(arg[6]);
    if (PyErr_Occurred()) return nullptr;
    status(mcf::check_attention(&c));
    const c10::Device device = ops.device();
    void *stream = stream_of(arg[8], device);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor made;
    int st;
    {
        const NoGil released;
        const Place place(device, stream);
        if (!out) { made = like(*q); c.out = rows(made); }
        int64_t bytes = 0;
        st = mcf_cache_attention_workspace(&c, &bytes);
        void *ws = nullptr;
        if (st == MCF_OK && bytes > 0) {
            try { // (a call without a workspace is not split)
                ws = workspace((size_t)bytes, (hipStream_t)stream, device);
            } catch (const c10::OutOfMemoryError &) {
            }
        }
        if (st == MCF_OK) st = mcf_cache_attention(&c, ws, ws ? bytes : 0, stream);
        if (ws) c10::hip::HIPCachingAllocator::raw_delete(ws);
        place.used(ops, {&made});
    }
    status(st);
    return wrap(out ? *out : made);
}

// Refusals become McfError, C++ exceptions of torch Python ones.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)> PyObject *entry(PyObject *, PyObject *const *arg, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        return F(arg, n);
    } catch (const Refused &r) {
        return r.text ? fail(r.status, r.text) : nullptr;
    }
    END_HANDLE_TH_ERRORS
}

#define MCF_METHOD(f, text) {#f, (PyCFunction)(void (*)(void))entry<f>, METH_FASTCALL, text}
PyMethodDef methods[] = {MCF_METHOD(norm_rotate, "mcf_norm_rotate on torch tensors"),
                         MCF_METHOD(norm_rotate_backward, "mcf_norm_rotate_backward on torch tensors"),
                         MCF_METHOD(append_cache, "mcf_cache_append on torch tensors"),
                         MCF_METHOD(cache_attention, "mcf_cache_attention on torch tensors"),
                         {"set_error", set_error, METH_O, "the exception type to raise"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mcf_cache", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__mcf_cache() { return PyModule_Create(&module); }
