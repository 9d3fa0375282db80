// Native argument marshalling for the Python binding (binding.py): the calls a decode loop makes, from torch tensors to
// the C ABI of libonela.so.
//
// What bounds it: host time.  Through ctypes a call cost 9 - 20 us of Python (shape tuples, dtype comparisons, one
// ctypes object per pointer, the current stream looked up through torch.cuda) against 2 - 10 us of kernel, so every
// call of a small batch waited for the host: a generation of the 8-beam fp32 workload took 99 us for 19 us of kernels.
// The same checks on the tensors' C++ objects take a fraction of a microsecond: 99 -> 33 us for that generation, 134 ->
// 72 us for the 128-beam one (four calls, 63 us of kernels).
//
// A call returns the library's status, or NOT_TAKEN when an argument is not what the fast path expects; binding.py
// then repeats the call through its own checks, which name the argument that is wrong.  Nothing is launched before all
// arguments have passed.  The library's functions are called through addresses handed over by binding.py, so this
// module works on whichever build of the library the process has loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>

#include "onela.h"

namespace {

constexpr long NOT_TAKEN = 1;

struct Api {
    decltype(&onela_export_chains) export_chains;
    decltype(&onela_init_shared_state) init_state;
    decltype(&onela_init_shared_states) init_states;
    decltype(&onela_prefill_shared_state) prefill;
    decltype(&onela_reorder_beams) reorder;
    decltype(&onela_select_beams) select;
    decltype(&onela_append_records) append;
    decltype(&onela_decode_step) decode;
    decltype(&onela_append_decode_step) append_decode;
    decltype(&onela_export_shared_state) export_state;
    decltype(&onela_release_request) release;
};
constexpr int API_FUNCTIONS = sizeof(Api) / sizeof(void*);

struct Caller {
    PyObject_HEAD
    Api api;
    onela_ctx* ctx;
    onela_config cfg;
    int64_t Hv;
    at::ScalarType rec, out;
};

// ---- arguments ----
bool int_of(PyObject* o, int32_t& v) {
    if (!PyLong_Check(o)) return false;
    const long x = PyLong_AsLong(o);
    if ((x == -1 && PyErr_Occurred()) || x != (int32_t)x) {
        PyErr_Clear();
        return false;
    }
    v = (int32_t)x;
    return true;
}

bool tensor_of(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, void*& p) {
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided) return false;
    const auto sizes = t.sizes();
    if (sizes.size() != shape.size()) return false;
    size_t i = 0;
    for (const int64_t n : shape)
        if (sizes[i++] != n) return false;
    if (!t.is_contiguous()) return false;
    p = t.data_ptr();
    return true;
}

bool stream_of(PyObject* o, void*& stream) {
    if (o == Py_None) {
        stream = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* raw = PyObject_GetAttrString(o, "cuda_stream");
    if (!raw) {
        PyErr_Clear();
        return false;
    }
    stream = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// beam width (and depth) of a request; 0 when it has none
int32_t width_of(const Caller* c, int32_t request, int32_t* depth = nullptr) {
    int32_t d = 0, w = 0;
    c->api.export_chains(c->ctx, request, nullptr, &d, &w, nullptr);
    if (depth) *depth = d;
    return w;
}

template <class F>
PyObject* call(F f) {
    onela_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}
PyObject* not_taken() { return PyLong_FromLong(NOT_TAKEN); }

// ---- the calls (positional arguments as in binding.py, the stream last) ----
PyObject* init_state(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r, l;
    void *S0, *s;
    if (n != 4 || !int_of(a[0], r) || !int_of(a[1], l) || !tensor_of(a[2], at::kFloat, {c->Hv, c->cfg.dv, c->cfg.dk}, S0) || !stream_of(a[3], s))
        return not_taken();
    return call([&] { return c->api.init_state(c->ctx, r, l, static_cast<const float*>(S0), s); });
}

PyObject* init_states(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r0, nr;
    void *S0, *s;
    if (n != 4 || !int_of(a[0], r0) || !int_of(a[1], nr) ||
        !tensor_of(a[2], at::kFloat, {nr, c->cfg.num_layers, c->Hv, c->cfg.dv, c->cfg.dk}, S0) || !stream_of(a[3], s))
        return not_taken();
    return call([&] { return c->api.init_states(c->ctx, r0, nr, static_cast<const float*>(S0), s); });
}

PyObject* prefill(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r, l;
    void *k, *v, *al, *be, *s;
    if (n != 7 || !int_of(a[0], r) || !int_of(a[1], l) || !THPVariable_Check(a[2])) return not_taken();
    const at::Tensor& kt = THPVariable_Unpack(a[2]);
    if (!kt.defined() || kt.dim() != 3 || kt.size(0) > INT32_MAX) return not_taken();
    const int64_t T = kt.size(0), H = c->cfg.num_heads;
    if (!tensor_of(a[2], c->rec, {T, H, c->cfg.dk}, k) || !tensor_of(a[3], c->rec, {T, H, c->cfg.dv}, v) ||
        !tensor_of(a[4], at::kFloat, {T, H}, al) || !tensor_of(a[5], at::kFloat, {T, H}, be) || !stream_of(a[6], s))
        return not_taken();
    return call([&] {
        return c->api.prefill(c->ctx, r, l, k, v, static_cast<const float*>(al), static_cast<const float*>(be), (int32_t)T, s);
    });
}

PyObject* reorder(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r0, nr, W;
    void *par = nullptr, *s;
    if (n != 5 || !int_of(a[0], r0) || !int_of(a[1], nr) || !int_of(a[3], W) ||
        (a[2] != Py_None && !tensor_of(a[2], at::kInt, {nr, W}, par)) || !stream_of(a[4], s))
        return not_taken();
    return call([&] { return c->api.reorder(c->ctx, r0, nr, static_cast<const int32_t*>(par), W, s); });
}

PyObject* select_beams(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r0, nr, C, W_new, depth;
    if (n != 10 || !int_of(a[0], r0) || !int_of(a[1], nr) || !int_of(a[4], C) || !int_of(a[5], W_new)) return not_taken();
    const int32_t W = width_of(c, r0, &depth), W_prev = depth >= 1 ? W : 1;
    void *bs, *lp, *par, *codes, *sc, *s;
    if (!tensor_of(a[2], at::kFloat, {nr, W_prev}, bs) || !tensor_of(a[3], at::kFloat, {nr, W_prev, C}, lp) ||
        !tensor_of(a[6], at::kInt, {nr, W_new}, par) || !tensor_of(a[7], at::kInt, {nr, W_new}, codes) ||
        !tensor_of(a[8], at::kFloat, {nr, W_new}, sc) || !stream_of(a[9], s))
        return not_taken();
    return call([&] {
        return c->api.select(c->ctx, r0, nr, static_cast<const float*>(bs), static_cast<const float*>(lp), C, W_new, static_cast<int32_t*>(par),
                             static_cast<int32_t*>(codes), static_cast<float*>(sc), s);
    });
}

struct Token {       // one decode call's records of a layer
    void *k, *v, *alpha, *beta;
};
bool token_of(const Caller* c, PyObject* const* a, int32_t nr, int32_t W, Token& t) {
    const int64_t Hk = c->cfg.num_heads;
    return tensor_of(a[0], c->rec, {nr, W, Hk, c->cfg.dk}, t.k) && tensor_of(a[1], c->rec, {nr, W, c->Hv, c->cfg.dv}, t.v) &&
           tensor_of(a[2], at::kFloat, {nr, W, c->Hv}, t.alpha) && tensor_of(a[3], at::kFloat, {nr, W, c->Hv}, t.beta);
}
bool query_of(const Caller* c, PyObject* const* a, int32_t nr, int32_t W, void*& q, void*& out) {
    return tensor_of(a[0], c->rec, {nr, W, (int64_t)c->cfg.num_heads, c->cfg.dk}, q) && tensor_of(a[1], c->out, {nr, W, c->Hv, c->cfg.dv}, out);
}

PyObject* append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r0, nr, l;
    Token t;
    void* s;
    if (n != 8 || !int_of(a[0], r0) || !int_of(a[1], nr) || !int_of(a[2], l) || !token_of(c, a + 3, nr, width_of(c, r0), t) || !stream_of(a[7], s))
        return not_taken();
    return call([&] {
        return c->api.append(c->ctx, r0, nr, l, t.k, t.v, static_cast<const float*>(t.alpha), static_cast<const float*>(t.beta), s);
    });
}

PyObject* decode(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r0, nr, l;
    void *q, *out, *s;
    if (n != 6 || !int_of(a[0], r0) || !int_of(a[1], nr) || !int_of(a[2], l) || !query_of(c, a + 3, nr, width_of(c, r0), q, out) || !stream_of(a[5], s))
        return not_taken();
    return call([&] { return c->api.decode(c->ctx, r0, nr, l, q, out, s); });
}

PyObject* append_decode(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r0, nr, l;
    if (n != 10 || !int_of(a[0], r0) || !int_of(a[1], nr) || !int_of(a[2], l)) return not_taken();
    const int32_t W = width_of(c, r0);
    Token t;
    void *q, *out, *s;
    if (!token_of(c, a + 3, nr, W, t) || !query_of(c, a + 7, nr, W, q, out) || !stream_of(a[9], s)) return not_taken();
    return call([&] {
        return c->api.append_decode(c->ctx, r0, nr, l, t.k, t.v, static_cast<const float*>(t.alpha), static_cast<const float*>(t.beta), q, out, s);
    });
}

PyObject* export_state(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r, l;
    void *S0, *s;
    if (n != 4 || !int_of(a[0], r) || !int_of(a[1], l) || !tensor_of(a[2], at::kFloat, {c->Hv, c->cfg.dv, c->cfg.dk}, S0) || !stream_of(a[3], s))
        return not_taken();
    return call([&] { return c->api.export_state(c->ctx, r, l, static_cast<float*>(S0), s); });
}

PyObject* release(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Caller*>(self);
    int32_t r;
    if (n != 1 || !int_of(a[0], r)) return not_taken();
    return PyLong_FromLong(c->api.release(c->ctx, r));
}

// ---- the operators without a context (positional arguments as in binding.py, the stream last) ----
struct Operators {
    PyObject_HEAD
    decltype(&onela_norm_rotate) norm_rotate;
    decltype(&onela_delta_rule) delta_rule;
    decltype(&onela_sample_tokens) sample_tokens;
};
constexpr int OPERATORS = 3;

// A tensor whose first dimension alone may be strided, on the current device; extents of -1 are read off it.
struct Rows {
    void* p = nullptr;
    int64_t stride = 0, size[4] = {0, 0, 0, 0};
};
bool rows_of(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, Rows& r) {
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || t.get_device() != c10::cuda::current_device()) return false;
    const auto sizes = t.sizes();
    const auto strides = t.strides();
    if (sizes.size() != shape.size()) return false;
    size_t i = 0;
    for (const int64_t n : shape) {
        if (n >= 0 && sizes[i] != n) return false;
        r.size[i] = sizes[i];
        ++i;
    }
    int64_t run = 1;
    for (size_t d = sizes.size() - 1; d > 0; --d) {
        if (sizes[d] != 1 && strides[d] != run) return false;
        run *= sizes[d];
    }
    // (a single row's stride means nothing: the next one that the library allows)
    const int64_t per = std::max<int64_t>(1, 16 / (int64_t)t.element_size());
    r.stride = sizes[0] > 1 ? strides[0] : (run + per - 1) / per * per;
    r.p = t.data_ptr();
    return true;
}
// A contiguous tensor or None (then `p` stays null)
bool dense_of(PyObject* o, at::ScalarType type, int64_t n, void*& p, int64_t* size = nullptr) {
    if (o == Py_None) return true;
    Rows r;
    if (!rows_of(o, type, {n}, r) || (r.size[0] > 1 && r.stride != 1)) return false;
    p = r.p;
    if (size) *size = r.size[0];
    return true;
}
bool float_of(PyObject* o, float& v) {
    if (!PyFloat_Check(o)) return false;
    v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
bool rec_of(PyObject* o, at::ScalarType& type, int32_t& code) {
    if (!THPVariable_Check(o)) return false;
    type = THPVariable_Unpack(o).scalar_type();
    code = type == at::kBFloat16 ? ONELA_DTYPE_BF16 : ONELA_DTYPE_F32;
    return type == at::kBFloat16 || type == at::kFloat;
}

// q, k, q_out, k_out, norm, eps, q_scale, q_weight, k_weight, positions, inv_freq, interleaved, stream
PyObject* norm_rotate(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Operators*>(self);
    onela_norm_rotate_args g = {};
    at::ScalarType t;
    Rows q, k, qo, ko;
    void *qw = nullptr, *kw = nullptr, *pos = nullptr, *freq = nullptr, *s;
    int64_t half = 0;
    if (n != 13 || !rec_of(a[0], t, g.dtype) || !rows_of(a[0], t, {-1, -1, -1}, q) || !rows_of(a[1], t, {q.size[0], -1, q.size[2]}, k) ||
        !rows_of(a[2], t, {q.size[0], q.size[1], q.size[2]}, qo) || !rows_of(a[3], t, {k.size[0], k.size[1], k.size[2]}, ko) || !int_of(a[4], g.norm) || g.norm < 0 ||
        !float_of(a[5], g.eps) || !float_of(a[6], g.q_scale) || !dense_of(a[7], at::kFloat, q.size[2], qw) || !dense_of(a[8], at::kFloat, q.size[2], kw) ||
        !dense_of(a[9], at::kInt, q.size[0], pos) || !dense_of(a[10], at::kFloat, -1, freq, &half) || !PyBool_Check(a[11]) || (a[9] == Py_None) != (a[10] == Py_None) ||
        ((qw || kw) && g.norm != ONELA_NORM_RMS) || q.size[1] > INT32_MAX || k.size[1] > INT32_MAX || q.size[2] > INT32_MAX || half > INT32_MAX / 2 || !stream_of(a[12], s))
        return not_taken();
    g.q_dev = q.p; g.k_dev = k.p; g.q_out_dev = qo.p; g.k_out_dev = ko.p;
    g.q_weight_dev = static_cast<const float*>(qw); g.k_weight_dev = static_cast<const float*>(kw);
    g.positions_dev = static_cast<const int32_t*>(pos); g.inv_freq_dev = static_cast<const float*>(freq);
    g.q_stride = q.stride; g.k_stride = k.stride; g.q_out_stride = qo.stride; g.k_out_stride = ko.stride;
    g.n_tokens = q.size[0]; g.num_q_heads = (int32_t)q.size[1]; g.num_k_heads = (int32_t)k.size[1]; g.head_dim = (int32_t)q.size[2];
    g.rotary_dim = (int32_t)(2 * half); g.interleaved = a[11] == Py_True;
    return call([&] { return c->norm_rotate(&g, s); });
}

// q, k, v, alpha, beta, states, out, starts, slots, fresh, max_tokens, status, stream
PyObject* delta_rule(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Operators*>(self);
    onela_delta_rule_args g = {};
    at::ScalarType t;
    Rows q, k, v, al, be, st, out;
    void *starts = nullptr, *slots = nullptr, *fresh = nullptr, *status = nullptr, *s;
    int64_t entries = 0;
    if (n != 13 || !rec_of(a[0], t, g.dtype) || !rows_of(a[0], t, {-1, -1, -1}, q) || !rows_of(a[1], t, {q.size[0], q.size[1], q.size[2]}, k) ||
        !rows_of(a[2], t, {q.size[0], -1, -1}, v) || !rows_of(a[3], at::kFloat, {q.size[0], v.size[1]}, al) || !rows_of(a[4], at::kFloat, {q.size[0], v.size[1]}, be) ||
        !rows_of(a[5], at::kFloat, {-1, v.size[1], v.size[2], q.size[2]}, st) || !rows_of(a[6], t, {q.size[0], v.size[1], v.size[2]}, out) ||
        !dense_of(a[7], at::kInt, -1, starts, &entries) || (a[7] != Py_None && entries < 1))
        return not_taken();
    const int64_t seqs = a[7] == Py_None ? q.size[0] : entries - 1;
    if (!dense_of(a[8], at::kInt, seqs, slots) || !dense_of(a[9], at::kInt, seqs, fresh) || !int_of(a[10], g.max_tokens) || !dense_of(a[11], at::kInt, 2, status) ||
        al.stride != be.stride || seqs > INT32_MAX || st.size[0] > INT32_MAX || q.size[1] > INT32_MAX || v.size[1] > INT32_MAX || q.size[2] > INT32_MAX ||
        v.size[2] > INT32_MAX || !stream_of(a[12], s))
        return not_taken();
    g.q_dev = q.p; g.k_dev = k.p; g.v_dev = v.p; g.out_dev = out.p;
    g.alpha_dev = static_cast<const float*>(al.p); g.beta_dev = static_cast<const float*>(be.p); g.states_dev = static_cast<float*>(st.p);
    g.starts_dev = static_cast<const int32_t*>(starts); g.slots_dev = static_cast<const int32_t*>(slots); g.fresh_dev = static_cast<const int32_t*>(fresh);
    g.status_dev = static_cast<int32_t*>(status);
    g.q_stride = q.stride; g.k_stride = k.stride; g.v_stride = v.stride; g.out_stride = out.stride; g.gate_stride = al.stride; g.state_stride = st.stride;
    g.n_tokens = q.size[0]; g.num_sequences = (int32_t)seqs; g.num_states = (int32_t)st.size[0];
    g.num_heads = (int32_t)q.size[1]; g.num_v_heads = (int32_t)v.size[1]; g.dk = (int32_t)q.size[2]; g.dv = (int32_t)v.size[2];
    return call([&] { return c->delta_rule(&g, s); });
}

// logits, uniforms, tokens_out, temperature, top_k, top_p, min_p, logprobs_out, stream
PyObject* sample_tokens(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    auto* c = reinterpret_cast<Operators*>(self);
    onela_sample_args g = {};
    at::ScalarType t;
    Rows x;
    void *u = nullptr, *tok = nullptr, *temp = nullptr, *k = nullptr, *p = nullptr, *m = nullptr, *lp = nullptr, *s;
    if (n != 9 || !rec_of(a[0], t, g.dtype) || !rows_of(a[0], t, {-1, -1}, x)) return not_taken();
    const int64_t R = x.size[0];
    if (a[1] == Py_None || a[2] == Py_None || !dense_of(a[1], at::kFloat, R, u) || !dense_of(a[2], at::kInt, R, tok) || !dense_of(a[3], at::kFloat, R, temp) ||
        !dense_of(a[4], at::kInt, R, k) || !dense_of(a[5], at::kFloat, R, p) || !dense_of(a[6], at::kFloat, R, m) || !dense_of(a[7], at::kFloat, R, lp) || R > INT32_MAX ||
        x.size[1] > INT32_MAX || !stream_of(a[8], s))
        return not_taken();
    g.logits_dev = x.p; g.uniforms_dev = static_cast<const float*>(u); g.tokens_out_dev = static_cast<int32_t*>(tok);
    g.temperature_dev = static_cast<const float*>(temp); g.top_p_dev = static_cast<const float*>(p); g.min_p_dev = static_cast<const float*>(m);
    g.top_k_dev = static_cast<const int32_t*>(k); g.logprobs_out_dev = static_cast<float*>(lp);
    g.logits_stride = R > 1 ? x.stride : x.size[1]; g.rows = (int32_t)R; g.vocab = (int32_t)x.size[1];
    return call([&] { return c->sample_tokens(&g, s); });
}

// ---- the types ----
int function_addresses(PyObject* fns, void** slots, int count) {
    if (PyTuple_GET_SIZE(fns) != count) {
        PyErr_SetString(PyExc_ValueError, "wrong number of library functions");
        return -1;
    }
    for (int i = 0; i < count; ++i) {
        slots[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(fns, i));
        if (PyErr_Occurred()) return -1;
    }
    return 0;
}
// Operators(function addresses in the order of its members)
int operators_init(PyObject* self, PyObject* args, PyObject*) {
    PyObject* fns;
    if (!PyArg_ParseTuple(args, "O!", &PyTuple_Type, &fns)) return -1;
    return function_addresses(fns, reinterpret_cast<void**>(&reinterpret_cast<Operators*>(self)->norm_rotate), OPERATORS);
}
// Caller(handle, config address, function addresses in the order of Api)
int caller_init(PyObject* self, PyObject* args, PyObject*) {
    auto* c = reinterpret_cast<Caller*>(self);
    unsigned long long handle, cfg;
    PyObject* fns;
    if (!PyArg_ParseTuple(args, "KKO!", &handle, &cfg, &PyTuple_Type, &fns)) return -1;
    if (function_addresses(fns, reinterpret_cast<void**>(&c->api), API_FUNCTIONS) != 0) return -1;
    c->ctx = reinterpret_cast<onela_ctx*>(handle);
    c->cfg = *reinterpret_cast<const onela_config*>(cfg);
    c->Hv = c->cfg.num_v_heads > 0 ? c->cfg.num_v_heads : c->cfg.num_heads;
    c->rec = c->cfg.rec_dtype == ONELA_DTYPE_BF16 ? at::kBFloat16 : at::kFloat;
    c->out = c->cfg.out_dtype == ONELA_DTYPE_BF16 ? at::kBFloat16 : at::kFloat;
    return 0;
}

// a C++ exception (from torch's side of a look-up) becomes a Python one
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    try {
        return F(self, args, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef caller_methods[] = {METHOD(init_state), METHOD(init_states),  METHOD(prefill), METHOD(reorder),       METHOD(select_beams),
                                METHOD(append),     METHOD(decode),       METHOD(append_decode), METHOD(export_state),  METHOD(release), {nullptr, nullptr, 0, nullptr}};
PyType_Slot caller_slots[] = {{Py_tp_init, reinterpret_cast<void*>(caller_init)},
                              {Py_tp_new, reinterpret_cast<void*>(PyType_GenericNew)},
                              {Py_tp_methods, caller_methods},
                              {0, nullptr}};
PyMethodDef operators_methods[] = {METHOD(norm_rotate), METHOD(delta_rule), METHOD(sample_tokens), {nullptr, nullptr, 0, nullptr}};
PyType_Slot operators_slots[] = {{Py_tp_init, reinterpret_cast<void*>(operators_init)},
                                 {Py_tp_new, reinterpret_cast<void*>(PyType_GenericNew)},
                                 {Py_tp_methods, operators_methods},
                                 {0, nullptr}};
PyType_Spec operators_spec = {"_onela_pycall.Operators", sizeof(Operators), 0, Py_TPFLAGS_DEFAULT, operators_slots};
PyType_Spec caller_spec = {"_onela_pycall.Caller", sizeof(Caller), 0, Py_TPFLAGS_DEFAULT, caller_slots};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_onela_pycall", nullptr, -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__onela_pycall() {
    PyObject *caller = PyType_FromSpec(&caller_spec), *operators = PyType_FromSpec(&operators_spec);
    PyObject* m = caller && operators ? PyModule_Create(&module_def) : nullptr;
    if (m && (PyModule_AddObjectRef(m, "Caller", caller) < 0 || PyModule_AddObjectRef(m, "Operators", operators) < 0 || PyModule_AddIntConstant(m, "NOT_TAKEN", NOT_TAKEN) < 0)) {
        Py_DECREF(m);
        m = nullptr;
    }
    Py_XDECREF(caller);
    Py_XDECREF(operators);
    return m;
}
