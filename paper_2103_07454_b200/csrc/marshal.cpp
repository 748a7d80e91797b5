// Argument marshalling of the operators around the step: torch tensors in, C ABI calls out.  A small call's kernels
// take a few microseconds; marshalling its arguments and allocating its outputs took 11 us a call in Python (norm, one
// pass forward and backward: 28 us).
// The library is not linked: `init` takes the addresses of its entry points, so that another build of it can be loaded.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>
#include <string>

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
PyMethodDef methods[] = {EG_ENTRY(init, 9), EG_ENTRY(residual_norm, 9), EG_ENTRY(residual_norm_backward, 10), EG_ENTRY(feed_forward, 7),
                         EG_ENTRY(feed_forward_backward, 8), EG_ENTRY(clip_gradients, 8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
