// Argument marshalling of the operators around the step: torch tensors in, C ABI calls out.  A small call's kernels
// take a few microseconds; marshalling its arguments and allocating its outputs took 11 us a call in Python (norm, one
// pass forward and backward: 28 us).
// The library is not linked: `init` takes the addresses of its entry points, so that another build of it can be loaded.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/eventgrad.h"

namespace {

struct Library {
    decltype(&eg_clip_gradients) clip;
    decltype(&eg_residual_norm) norm;
    decltype(&eg_residual_norm_backward) norm_backward;
    decltype(&eg_residual_norm_workspace) norm_workspace;
    decltype(&eg_feed_forward) ffn;
    decltype(&eg_feed_forward_backward) ffn_backward;
    decltype(&eg_feed_forward_saved_bytes) ffn_saved;
    decltype(&eg_feed_forward_workspace) ffn_workspace;
    decltype(&eg_embedding) embed;
    decltype(&eg_embedding_backward) embed_backward;
    decltype(&eg_embedding_workspace) embed_workspace;
    decltype(&eg_head_norm) heads;
    decltype(&eg_head_norm_backward) heads_backward;
    decltype(&eg_head_norm_workspace) heads_workspace;
    decltype(&eg_orthogonalise) ortho;
    decltype(&eg_orthogonalise_workspace) ortho_workspace;
} lib;
PyObject* error_class = nullptr;

struct Refused {                                   // becomes an EventGradError
    std::string text;
};

int type_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return EG_F32;
        case at::kBFloat16: return EG_BF16;
        case at::kHalf: return EG_F16;
        default: return -1;
    }
}

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) throw Refused{std::string(what) + ": expected a tensor, got " + Py_TYPE(o)->tp_name};
    return THPVariable_Unpack(o);
}

const at::Tensor& on_device(const at::Tensor& t) {
    if (!t.is_cuda()) throw Refused{"no CUDA device: this library has no CPU path"};
    return t;
}

// The calls take no part in autograd.  Results without a graph where one is expected would be gradients lost without a word.
const at::Tensor& plain(const at::Tensor& t, const char* what) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
        throw Refused{std::string(what) + " requires a gradient, but the operators take no part in autograd: call them under "
                                          "torch.no_grad(), and the *_backward calls for the gradients"};
    return t;
}

// What a call's tensors have in common.
struct Kind {
    at::ScalarType type;
    at::Device device;
    at::Tensor empty(at::IntArrayRef sizes) const { return at::detail::empty_cuda(sizes, type, device, c10::nullopt); }
    at::Tensor bytes(int64_t n) const { return at::detail::empty_cuda({n}, at::kByte, device, c10::nullopt); }
};

// (pointer, replica stride, row stride) of a [P, rows, columns] or [P, columns] tensor, or of None.
eg_matrix given(PyObject* o, at::IntArrayRef sizes, const Kind& k, const char* what) {
    if (o == Py_None) return eg_matrix{};
    const at::Tensor& t = tensor(o, what);
    if (t.sizes() != sizes || t.scalar_type() != k.type || t.device() != k.device) {
        std::string s = std::string(what) + ": expected [";
        for (int64_t n : sizes) s += std::to_string(n) + ", ";
        s += std::string("] ") + c10::toString(k.type) + " on " + k.device.str() + ", got [";
        for (int64_t n : t.sizes()) s += std::to_string(n) + ", ";
        throw Refused{s + "] " + c10::toString(t.scalar_type()) + " on " + t.device().str()};
    }
    plain(t, what);
    const auto st = t.strides();
    if (st.back() != 1 && sizes.back() > 1) throw Refused{std::string(what) + ": the last dimension must be contiguous"};
    return eg_matrix{t.data_ptr(), st[0], sizes.size() == 3 ? st[1] : 0};
}
eg_matrix made(const at::Tensor& t) { return eg_matrix{t.data_ptr(), t.stride(0), t.dim() == 3 ? t.stride(1) : 0}; }

// Owned references that a result is put together from.
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* same(PyObject* o) { Py_INCREF(o); return o; }
PyObject* none() { Py_RETURN_NONE; }
template <typename... O> PyObject* tuple(O... items) {
    PyObject* all[] = {items...};
    bool ok = true;
    for (PyObject* o : all) ok = ok && o;
    PyObject* r = ok ? PyTuple_New(sizeof...(items)) : nullptr;
    Py_ssize_t i = 0;
    for (PyObject* o : all) {
        if (r) PyTuple_SET_ITEM(r, i++, o);
        else Py_XDECREF(o);
    }
    return r;
}

// A call into the library without the interpreter's lock; a status other than EG_OK is the function's result.
template <typename F> eg_status unlocked(F&& f) {
    eg_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return st;
}

// An entry point that builds of the library from before it lack.
template <typename F> void needed(F* f, const char* what) {
    if (!f) throw Refused{std::string(what) + " is not in this build of the library: build it with `python -m paper_2103_07454_b200.build`"};
}

// Every entry: the number of arguments is checked, no C++ exception leaves.
template <PyObject* (*F)(PyObject* const*), int N> PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Refused& r) {
        PyErr_SetString(error_class, r.text.c_str());
    } catch (const c10::OutOfMemoryError& e) {
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type);
        Py_XDECREF(torch);
    } catch (const c10::Error& e) {
        PyErr_SetString(error_class, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{"expected a number"};
    }
    return v;
}
long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{"expected an integer"};
    }
    return v;
}

// ------------------------------------------------------------------------------- the norm
struct NormCall {
    const at::Tensor& r;
    Kind k;
    c10::cuda::CUDAGuard guard;
    eg_residual_norm_args q{};

    NormCall(const at::Tensor& residual, PyObject* y, PyObject* const* vectors, PyObject* eps, const char* what)
        : r(on_device(shaped(residual, what))), k{r.scalar_type(), r.device()}, guard(k.device) {
        plain(r, "residual");
        q.P = r.size(0); q.rows = r.size(1); q.width = r.size(2);
        q.dtype = type_of(r);
        q.eps = number(eps);
        q.y = given(y, r.sizes(), k, "y");
        q.residual = eg_matrix{r.data_ptr(), r.stride(0), r.stride(1)};
        if (r.stride(2) != 1 && q.width > 1) throw Refused{"residual: the last dimension must be contiguous"};
        const int64_t vec[] = {q.P, q.width};
        q.w_post = given(vectors[0], vec, k, "w_post");
        q.gate = given(vectors[1], vec, k, "gate");
        q.scale = given(vectors[2], vec, k, "scale");
        q.w_pre = given(vectors[3], vec, k, "w_pre");
    }
    static const at::Tensor& shaped(const at::Tensor& t, const char* what) {
        if (t.dim() != 3 || type_of(t) < 0) throw Refused{std::string(what) + ": residual must be [P, rows, width] fp32, bf16 or fp16"};
        return t;
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(k.device.index()).stream(); }
};

// y, residual, w_post, gate, scale, w_pre, eps, residual_out, out
PyObject* residual_norm(PyObject* const* a) {
    NormCall c(tensor(a[1], "residual"), a[0], a + 2, a[6], "residual_norm");
    at::Tensor res, out;
    c.q.residual_out = a[7] != Py_None ? given(a[7], c.r.sizes(), c.k, "residual_out") : made(res = c.k.empty(c.r.sizes()));
    if (a[8] != Py_None) c.q.out = given(a[8], c.r.sizes(), c.k, "out");
    else if (a[5] != Py_None) c.q.out = made(out = c.k.empty(c.r.sizes()));
    if (c.q.rows > 0) {
        void* s = c.stream();
        const eg_status st = unlocked([&] { return lib.norm(&c.q, s); });
        if (st != EG_OK) return PyLong_FromLong(st);
    }
    return tuple(res.defined() ? wrap(res) : same(a[7]), out.defined() ? wrap(out) : same(a[8]));
}

// d_residual_out, d_out, y, residual, w_post, gate, scale, w_pre, eps, d_weights (tuple of four, or None)
PyObject* residual_norm_backward(PyObject* const* a) {
    NormCall c(tensor(a[3], "residual"), a[2], a + 4, a[8], "residual_norm_backward");
    c.q.d_residual_out = given(a[0], c.r.sizes(), c.k, "d_residual_out");
    c.q.d_out = given(a[1], c.r.sizes(), c.k, "d_out");
    const int64_t vec[] = {c.q.P, c.q.width};
    at::Tensor fresh[4];
    eg_matrix* to[] = {&c.q.d_w_post, &c.q.d_gate, &c.q.d_scale, &c.q.d_w_pre};
    static const char* const names[] = {"d_w_post", "d_gate", "d_scale", "d_w_pre"};
    for (int i = 0; i < 4; ++i) {
        if (a[9] != Py_None) *to[i] = given(PyTuple_GET_ITEM(a[9], i), vec, c.k, names[i]);
        else if (a[4 + i] != Py_None) *to[i] = made(fresh[i] = c.k.empty(vec));
    }
    at::Tensor dy, dr = c.k.empty(c.r.sizes());
    if (a[2] != Py_None) c.q.dy = made(dy = c.k.empty(c.r.sizes()));
    c.q.d_residual = made(dr);
    c.q.workspace_bytes = lib.norm_workspace(c.q.P, c.q.width);
    const at::Tensor workspace = c.k.bytes(c.q.workspace_bytes);
    c.q.workspace = workspace.data_ptr();
    if (c.q.rows > 0) {
        void* s = c.stream();
        const eg_status st = unlocked([&] { return lib.norm_backward(&c.q, s); });
        if (st != EG_OK) return PyLong_FromLong(st);
    } else {
        for (int i = 0; i < 4; ++i) {
            if (fresh[i].defined()) fresh[i].zero_();
            else if (a[9] != Py_None && PyTuple_GET_ITEM(a[9], i) != Py_None) at::Tensor(tensor(PyTuple_GET_ITEM(a[9], i), names[i])).detach().zero_();
        }
    }
    PyObject* weights = a[9] != Py_None ? same(a[9])
                                        : tuple(fresh[0].defined() ? wrap(fresh[0]) : none(), fresh[1].defined() ? wrap(fresh[1]) : none(),
                                                fresh[2].defined() ? wrap(fresh[2]) : none(), fresh[3].defined() ? wrap(fresh[3]) : none());
    return tuple(dy.defined() ? wrap(dy) : none(), wrap(dr), weights);
}

// ------------------------------------------------------------------------------- the feed-forward block
struct FfnCall {
    const at::Tensor& x;
    Kind k;
    c10::cuda::CUDAGuard guard;
    eg_feed_forward_args q{};
    int64_t up[3], down[3];

    FfnCall(PyObject* const* a, const char* what)                  // x, w_gate, w_up, w_down, activation
        : x(on_device(shaped(a, what))), k{x.scalar_type(), x.device()}, guard(k.device) {
        q.P = x.size(0); q.rows = x.size(1); q.d_model = x.size(2);
        q.d_ff = THPVariable_Unpack(a[1]).size(1);
        q.dtype = type_of(x);
        q.activation = integer(a[4]);
        up[0] = down[0] = q.P; up[1] = down[2] = q.d_ff; up[2] = down[1] = q.d_model;
        q.x = given(a[0], x.sizes(), k, "x");
        q.w_gate = given(a[1], up, k, "w_gate");
        q.w_up = given(a[2], up, k, "w_up");
        q.w_down = given(a[3], down, k, "w_down");
    }
    static const at::Tensor& shaped(PyObject* const* a, const char* what) {
        const at::Tensor &t = tensor(a[0], "x"), &g = tensor(a[1], "w_gate");
        if (t.dim() != 3 || g.dim() != 3 || type_of(t) < 0)
            throw Refused{std::string(what) + ": x must be [P, rows, d_model] and w_gate [P, d_ff, d_model], fp32, bf16 or fp16"};
        return t;
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(k.device.index()).stream(); }
};

// x, w_gate, w_up, w_down, activation, save, out
PyObject* feed_forward(PyObject* const* a) {
    FfnCall c(a, "feed_forward");
    for (int i = 1; i < 4; ++i)
        if (a[i] == Py_None) throw Refused{"feed_forward: three weights"};
    at::Tensor out, saved, workspace;
    c.q.y = a[6] != Py_None ? given(a[6], c.x.sizes(), c.k, "out") : made(out = c.k.empty(c.x.sizes()));
    const bool save = a[5] == Py_True;
    if (save) {
        c.q.saved_bytes = lib.ffn_saved(&c.q);
        c.q.saved = (saved = c.k.bytes(c.q.saved_bytes)).data_ptr();
    }
    if (c.q.rows > 0) {
        const int64_t bytes = lib.ffn_workspace(&c.q, 0);
        void* w = bytes ? (workspace = c.k.bytes(bytes)).data_ptr() : nullptr;
        void* s = c.stream();
        const eg_status st = unlocked([&] { return lib.ffn(&c.q, w, bytes, s); });
        if (st != EG_OK) return PyLong_FromLong(st);
    }
    PyObject* y = out.defined() ? wrap(out) : same(a[6]);
    return save ? tuple(y, wrap(saved)) : y;
}

// x, w_gate, w_up, w_down, activation, dy, saved, d_weights (tuple of three, or None)
PyObject* feed_forward_backward(PyObject* const* a) {
    FfnCall c(a, "feed_forward_backward");
    c.q.dy = given(a[5], c.x.sizes(), c.k, "dy");
    const at::Tensor& saved = tensor(a[6], "saved");
    if (saved.device() != c.k.device || saved.scalar_type() != at::kByte || !saved.is_contiguous())
        throw Refused{"feed_forward_backward: saved is what feed_forward(..., save=True) returned"};
    c.q.saved = saved.data_ptr();
    c.q.saved_bytes = saved.numel();
    at::Tensor fresh[3];
    eg_matrix* to[] = {&c.q.d_gate, &c.q.d_up, &c.q.d_down};
    static const char* const names[] = {"d_gate", "d_up", "d_down"};
    for (int i = 0; i < 3; ++i) {
        const at::IntArrayRef sizes(i == 2 ? c.down : c.up, 3);
        *to[i] = a[7] != Py_None ? given(PyTuple_GET_ITEM(a[7], i), sizes, c.k, names[i]) : made(fresh[i] = c.k.empty(sizes));
    }
    const at::Tensor dx = c.k.empty(c.x.sizes());
    c.q.dx = made(dx);
    const int64_t bytes = lib.ffn_workspace(&c.q, 1);
    const at::Tensor workspace = c.k.bytes(bytes);
    void *w = workspace.data_ptr(), *s = c.stream();
    const eg_status st = unlocked([&] { return lib.ffn_backward(&c.q, w, bytes, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    return tuple(wrap(dx), a[7] != Py_None ? same(a[7]) : tuple(wrap(fresh[0]), wrap(fresh[1]), wrap(fresh[2])));
}

// ------------------------------------------------------------------------------- tokens
// [P, rows] whole numbers on the device, of any strides: (pointer, bytes, replica stride, stride).
struct Numbers {
    const void* data;
    int64_t bytes, replica_stride, stride;
};
Numbers numbers(const at::Tensor& t, int64_t P, int64_t rows, const Kind& k, const char* what) {
    if (t.dim() != 2 || t.size(0) != P || t.size(1) != rows || (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) || t.device() != k.device)
        throw Refused{std::string(what) + ": expected [" + std::to_string(P) + ", " + std::to_string(rows) + "] int32 or int64 on " + k.device.str()};
    return Numbers{t.data_ptr(), t.scalar_type() == at::kInt ? 4 : 8, t.stride(0), t.stride(1)};
}

void* stream_of(const Kind& k) { return c10::cuda::getCurrentCUDAStream(k.device.index()).stream(); }

void set_tokens(eg_embedding_args& q, const at::Tensor& tokens, const Kind& k, const char* what) {
    if (tokens.dim() != 2) throw Refused{std::string(what) + ": tokens must be [P, rows]"};
    q.P = tokens.size(0);
    q.rows = tokens.size(1);
    const Numbers n = numbers(tokens, q.P, q.rows, k, "tokens");
    q.tokens = n.data; q.token_bytes = n.bytes; q.token_replica_stride = n.replica_stride; q.token_stride = n.stride;
}

// tokens, weight, scale, out
PyObject* embedding(PyObject* const* a) {
    needed(lib.embed, "eg_embedding");
    const at::Tensor &tokens = tensor(a[0], "tokens"), &w = on_device(tensor(a[1], "weight"));
    if (w.dim() != 3 || type_of(w) < 0) throw Refused{"embedding: weight must be [P, vocabulary, width] fp32, bf16 or fp16"};
    const Kind k{w.scalar_type(), w.device()};
    const c10::cuda::CUDAGuard guard(k.device);
    eg_embedding_args q{};
    set_tokens(q, tokens, k, "embedding");
    q.vocabulary = w.size(1); q.width = w.size(2); q.dtype = type_of(w);
    q.scale = number(a[2]);
    const int64_t table[] = {q.P, q.vocabulary, q.width}, sizes[] = {q.P, q.rows, q.width};
    q.weight = given(a[1], table, k, "weight");
    at::Tensor out;
    q.out = a[3] != Py_None ? given(a[3], sizes, k, "out") : made(out = k.empty(sizes));
    void* s = stream_of(k);
    const eg_status st = unlocked([&] { return lib.embed(&q, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    return out.defined() ? wrap(out) : same(a[3]);
}

// dy, tokens, vocabulary, scale, d_weight, accumulate
PyObject* embedding_backward(PyObject* const* a) {
    needed(lib.embed_backward, "eg_embedding_backward");
    const at::Tensor &dy = on_device(tensor(a[0], "dy")), &tokens = tensor(a[1], "tokens");
    if (dy.dim() != 3 || type_of(dy) < 0) throw Refused{"embedding_backward: dy must be [P, rows, width] fp32, bf16 or fp16"};
    const Kind k{dy.scalar_type(), dy.device()};
    const c10::cuda::CUDAGuard guard(k.device);
    eg_embedding_args q{};
    set_tokens(q, tokens, k, "embedding_backward");
    q.width = dy.size(2); q.dtype = type_of(dy);
    q.scale = number(a[3]);
    q.accumulate = a[5] == Py_True;
    const int64_t sizes[] = {q.P, q.rows, q.width};
    q.dy = given(a[0], sizes, k, "dy");
    at::Tensor fresh;
    if (a[4] != Py_None) {
        const at::Tensor& d = tensor(a[4], "d_weight");
        if (d.dim() != 3 || (a[2] != Py_None && d.size(1) != integer(a[2])))
            throw Refused{"embedding_backward: d_weight must be [P, vocabulary, width]"};
        q.vocabulary = d.size(1);
        const int64_t table[] = {q.P, q.vocabulary, q.width};
        q.d_weight = given(a[4], table, k, "d_weight");
    } else {
        if (q.accumulate) throw Refused{"embedding_backward: accumulate adds to a given d_weight"};
        if (a[2] == Py_None) throw Refused{"embedding_backward: give d_weight or the vocabulary's size"};
        q.vocabulary = integer(a[2]);
        if (q.vocabulary < 1) throw Refused{"embedding_backward: the vocabulary has at least one row"};
        const int64_t table[] = {q.P, q.vocabulary, q.width};
        q.d_weight = made(fresh = k.empty(table));
    }
    const int64_t bytes = lib.embed_workspace(&q);
    const at::Tensor workspace = k.bytes(bytes);
    void *w = workspace.data_ptr(), *s = stream_of(k);
    const eg_status st = unlocked([&] { return lib.embed_backward(&q, w, bytes, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    return fresh.defined() ? wrap(fresh) : same(a[4]);
}

// ------------------------------------------------------------------------------- heads
eg_heads given_heads(PyObject* o, at::IntArrayRef sizes, const Kind& k, const char* what) {
    if (o == Py_None) return eg_heads{};
    const at::Tensor& t = tensor(o, what);
    if (t.sizes() != sizes || t.scalar_type() != k.type || t.device() != k.device) {
        std::string s = std::string(what) + ": expected [";
        for (int64_t n : sizes) s += std::to_string(n) + ", ";
        throw Refused{s + "] " + c10::toString(k.type) + " on " + k.device.str()};
    }
    plain(t, what);
    if (t.stride(3) != 1 && sizes[3] > 1) throw Refused{std::string(what) + ": the last dimension must be contiguous"};
    return eg_heads{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}
eg_heads made_heads(const at::Tensor& t) { return eg_heads{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }

struct HeadsCall {
    const at::Tensor& q_;
    Kind k;
    c10::cuda::CUDAGuard guard;
    eg_head_norm_args q{};
    int64_t q_sizes[4], k_sizes[4], vec[2];
    bool keys;

    // q, k, w_q, w_k, positions, rotary, base, interleaved, eps
    HeadsCall(PyObject* const* a, const char* what) : q_(on_device(shaped(a, what))), k{q_.scalar_type(), q_.device()}, guard(k.device) {
        keys = a[1] != Py_None;
        q.P = q_.size(0); q.rows = q_.size(1); q.q_heads = q_.size(2); q.width = q_.size(3);
        q.k_heads = keys ? THPVariable_Unpack(a[1]).size(2) : 0;
        q.dtype = type_of(q_);
        const int64_t qs[] = {q.P, q.rows, q.q_heads, q.width}, ks[] = {q.P, q.rows, q.k_heads, q.width};
        std::memcpy(q_sizes, qs, sizeof qs);
        std::memcpy(k_sizes, ks, sizeof ks);
        vec[0] = q.P; vec[1] = q.width;
        q.q = given_heads(a[0], q_sizes, k, "q");
        q.k = given_heads(a[1], k_sizes, k, "k");
        q.w_q = given(a[2], vec, k, "w_q");
        q.w_k = given(a[3], vec, k, "w_k");
        if (a[4] != Py_None) {
            const Numbers n = numbers(tensor(a[4], "positions"), q.P, q.rows, k, "positions");
            q.positions = n.data; q.position_bytes = n.bytes; q.position_replica_stride = n.replica_stride; q.position_stride = n.stride;
        }
        q.rotary = a[5] == Py_None ? q.width / 2 * 2 : integer(a[5]);
        q.base = number(a[6]);
        q.interleaved = a[7] == Py_True;
        q.eps = number(a[8]);
    }
    static const at::Tensor& shaped(PyObject* const* a, const char* what) {
        const at::Tensor& t = tensor(a[0], "q");
        if (t.dim() != 4 || type_of(t) < 0) throw Refused{std::string(what) + ": q must be [P, rows, heads, width] fp32, bf16 or fp16"};
        if (a[1] != Py_None && tensor(a[1], "k").dim() != 4) throw Refused{std::string(what) + ": k must be [P, rows, heads, width]"};
        return t;
    }
};

// q, k, w_q, w_k, positions, rotary, base, interleaved, eps, q_out, k_out
PyObject* head_norm(PyObject* const* a) {
    needed(lib.heads, "eg_head_norm");
    HeadsCall c(a, "head_norm");
    if (!c.keys && a[10] != Py_None) throw Refused{"head_norm: k_out without k"};
    at::Tensor q_out, k_out;
    c.q.q_out = a[9] != Py_None ? given_heads(a[9], c.q_sizes, c.k, "q_out") : made_heads(q_out = c.k.empty(c.q_sizes));
    if (a[10] != Py_None) c.q.k_out = given_heads(a[10], c.k_sizes, c.k, "k_out");
    else if (c.keys) c.q.k_out = made_heads(k_out = c.k.empty(c.k_sizes));
    void* s = stream_of(c.k);
    const eg_status st = unlocked([&] { return lib.heads(&c.q, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    return tuple(q_out.defined() ? wrap(q_out) : same(a[9]), k_out.defined() ? wrap(k_out) : same(a[10]));
}

// q, k, w_q, w_k, positions, rotary, base, interleaved, eps, dq_out, dk_out, dq, dk, d_weights (tuple of two, or None)
PyObject* head_norm_backward(PyObject* const* a) {
    needed(lib.heads_backward, "eg_head_norm_backward");
    HeadsCall c(a, "head_norm_backward");
    if (!c.keys && (a[10] != Py_None || a[12] != Py_None)) throw Refused{"head_norm_backward: dk_out or dk without k"};
    if (a[9] == Py_None || (c.keys && a[10] == Py_None)) throw Refused{"head_norm_backward: the gradients of both outputs are needed"};
    c.q.dq_out = given_heads(a[9], c.q_sizes, c.k, "dq_out");
    c.q.dk_out = given_heads(a[10], c.k_sizes, c.k, "dk_out");
    at::Tensor dq, dk, fresh[2];
    c.q.dq = a[11] != Py_None ? given_heads(a[11], c.q_sizes, c.k, "dq") : made_heads(dq = c.k.empty(c.q_sizes));
    if (a[12] != Py_None) c.q.dk = given_heads(a[12], c.k_sizes, c.k, "dk");
    else if (c.keys) c.q.dk = made_heads(dk = c.k.empty(c.k_sizes));
    eg_matrix* to[] = {&c.q.d_w_q, &c.q.d_w_k};
    static const char* const names[] = {"d_w_q", "d_w_k"};
    for (int i = 0; i < 2; ++i) {
        if (a[13] != Py_None) *to[i] = given(PyTuple_GET_ITEM(a[13], i), c.vec, c.k, names[i]);
        else if (a[2 + i] != Py_None) *to[i] = made(fresh[i] = c.k.empty(c.vec));
    }
    const int64_t bytes = lib.heads_workspace(&c.q);
    const at::Tensor workspace = c.k.bytes(bytes);
    void *w = workspace.data_ptr(), *s = stream_of(c.k);
    const eg_status st = unlocked([&] { return lib.heads_backward(&c.q, w, bytes, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    PyObject* weights = a[13] != Py_None ? same(a[13]) : tuple(fresh[0].defined() ? wrap(fresh[0]) : none(), fresh[1].defined() ? wrap(fresh[1]) : none());
    return tuple(dq.defined() ? wrap(dq) : same(a[11]), dk.defined() ? wrap(dk) : same(a[12]), weights);
}

// ------------------------------------------------------------------------------- matrices
// The i-th of a tuple, or None.
PyObject* item(PyObject* o, Py_ssize_t i) { return o == Py_None ? Py_None : PyTuple_GET_ITEM(o, i); }

// grads, out, velocity, velocity_out (tuples or None), momentum, nesterov, steps, coefficients (tuple of numbers, or None), scales (tuple)
PyObject* orthogonalise(PyObject* const* a) {
    needed(lib.ortho, "eg_orthogonalise");
    const Py_ssize_t count = PyTuple_GET_SIZE(a[0]);
    if (count == 0) return PyTuple_New(0);
    const at::Tensor& first = on_device(tensor(PyTuple_GET_ITEM(a[0], 0), "grads"));
    if (first.dim() != 3 || type_of(first) < 0) throw Refused{"orthogonalise: a gradient must be [P, rows, columns] fp32, bf16 or fp16"};
    const Kind k{first.scalar_type(), first.device()}, wide{at::kFloat, k.device};
    const at::Tensor& first_out = a[1] == Py_None ? first : tensor(PyTuple_GET_ITEM(a[1], 0), "out");
    const Kind result{first_out.scalar_type(), k.device};
    const c10::cuda::CUDAGuard guard(k.device);
    eg_orthogonalise_args q{};
    q.P = first.size(0); q.count = count; q.dtype = type_of(first); q.out_dtype = type_of(first_out);
    q.momentum = number(a[4]);
    q.nesterov = a[5] == Py_True;
    q.steps = integer(a[6]);
    std::vector<double> coefficients;
    if (a[7] != Py_None) {
        if (q.steps < 1 || PyTuple_GET_SIZE(a[7]) != 3 * q.steps) throw Refused{"orthogonalise: three coefficients, or three for every step"};
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[7]); ++i) coefficients.push_back(number(PyTuple_GET_ITEM(a[7], i)));
        q.coefficients = coefficients.data();
    }
    std::vector<eg_orthogonal_matrix> all(count);
    q.matrices = all.data();
    std::vector<const void*> written;
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor& g = tensor(PyTuple_GET_ITEM(a[0], i), "grads");
        if (g.dim() != 3) throw Refused{"orthogonalise: a gradient must be [P, rows, columns]"};
        const int64_t sizes[] = {q.P, g.size(1), g.size(2)};
        eg_orthogonal_matrix& m = all[i];
        m.rows = sizes[1]; m.columns = sizes[2];
        m.scale = number(PyTuple_GET_ITEM(a[8], i));
        m.grad = given(PyTuple_GET_ITEM(a[0], i), sizes, k, "grads");
        m.out = a[1] == Py_None ? m.grad : given(PyTuple_GET_ITEM(a[1], i), sizes, result, "out");
        m.velocity = given(item(a[2], i), sizes, wide, "velocity");
        m.velocity_out = given(item(a[3], i), sizes, wide, "velocity_out");
        written.push_back(m.out.data);
        if (m.velocity.data) written.push_back(m.velocity_out.data ? m.velocity_out.data : m.velocity.data);
    }
    std::sort(written.begin(), written.end());
    if (std::adjacent_find(written.begin(), written.end()) != written.end()) throw Refused{"orthogonalise: two results lie on one another"};
    const int64_t bytes = lib.ortho_workspace(&q);
    const at::Tensor workspace = k.bytes(bytes);
    void *w = workspace.data_ptr(), *s = stream_of(k);
    const eg_status st = unlocked([&] { return lib.ortho(&q, w, bytes, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    return same(a[1] == Py_None ? a[0] : a[1]);
}

// ------------------------------------------------------------------------------- clipping
// context, P, replica_stride, grads, out, max_norm, flags, norms
PyObject* clip_gradients(PyObject* const* a) {
    const at::Tensor &g = plain(tensor(a[3], "grads"), "grads"), &out = a[4] == Py_None ? g : plain(tensor(a[4], "out"), "out");
    const int64_t P = integer(a[1]), sizes[] = {P, integer(a[2])};
    const int type = type_of(g);
    const char* wrong = nullptr;
    if (type < 0 || out.scalar_type() != at::kFloat) wrong = "grads are fp32, bf16 or fp16, the result is fp32";
    else if (!g.is_cuda() || g.device() != out.device()) wrong = "grads and out lie on the device";
    else if (!g.is_contiguous() || !out.is_contiguous()) wrong = "grads and out are contiguous";
    else if (g.sizes() != at::IntArrayRef(sizes, 2) || out.sizes() != g.sizes()) wrong = "grads and out are [P, replica_stride]";
    at::Tensor norms;
    if (!wrong) {
        if (a[7] == Py_None) norms = at::detail::empty_cuda({P}, at::kFloat, out.device(), c10::nullopt);
        else norms = tensor(a[7], "norms");
        if (norms.device() != out.device() || norms.scalar_type() != at::kFloat || !norms.is_contiguous() || norms.numel() != P)
            wrong = "norms is [P] fp32 on the device, contiguous";
    }
    if (wrong) {
        PyErr_SetString(PyExc_AssertionError, wrong);
        return nullptr;
    }
    const c10::cuda::CUDAGuard guard(out.device());
    void* s = c10::cuda::getCurrentCUDAStream(out.device().index()).stream();
    eg_ctx* ctx = reinterpret_cast<eg_ctx*>(integer(a[0]));
    const double max_norm = number(a[5]);
    const int flags = (int)integer(a[6]);
    const void* from = g.data_ptr();
    float *to = static_cast<float*>(out.data_ptr()), *n = static_cast<float*>(norms.data_ptr());
    const eg_status st = unlocked([&] { return lib.clip(ctx, from, type, max_norm, flags, to, n, s); });
    if (st != EG_OK) return PyLong_FromLong(st);
    return a[7] == Py_None ? wrap(norms) : same(a[7]);
}

// error class, then the entry points' addresses in the order of Library
PyObject* init(PyObject* const* a) {
    Py_INCREF(a[0]);
    Py_XSETREF(error_class, a[0]);
    void* at[sizeof(Library) / sizeof(void*)];
    for (size_t i = 0; i < sizeof(at) / sizeof(void*); ++i) at[i] = reinterpret_cast<void*>(integer(a[1 + i]));
    std::memcpy(&lib, at, sizeof lib);
    return none();
}

#define EG_ENTRY(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {EG_ENTRY(init, 1 + sizeof(Library) / sizeof(void*)), EG_ENTRY(residual_norm, 9), EG_ENTRY(residual_norm_backward, 10), EG_ENTRY(feed_forward, 7),
                         EG_ENTRY(feed_forward_backward, 8), EG_ENTRY(clip_gradients, 8), EG_ENTRY(embedding, 4), EG_ENTRY(embedding_backward, 6),
                         EG_ENTRY(head_norm, 11), EG_ENTRY(head_norm_backward, 14), EG_ENTRY(orthogonalise, 9), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
