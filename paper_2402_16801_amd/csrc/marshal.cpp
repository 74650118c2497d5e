// Tensors to the C ABI: checks shapes, types and strides, allocates outputs and workspaces, fills the argument
// structure and makes the call.  It is the inner half of memory.py, in C++ because a call for one token of a few
// environments takes a few microseconds on the GPU and the same checks take three to six times that in
// Python.  No arithmetic here.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/impl/HIPGuardImplMasqueradingAsCUDA.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/GradMode.h>
#include <c10/util/Exception.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <initializer_list>
#include <sstream>
#include <stdexcept>
#include <string>

#include "../../include/craftax.h"

namespace {

using at::Tensor;

struct Refusal : std::runtime_error {
    using std::runtime_error::runtime_error;
};

PyObject* g_error = nullptr;      // CraftaxError
PyObject* g_no_memory = nullptr;  // torch.OutOfMemoryError

// The entry points of the loaded library (the release or the debug one), set by bind().
struct Library {
    int (*conv)(const craftax_conv_args*, void*);
    int (*conv_backward)(const craftax_conv_args*, void*);
    size_t (*conv_workspace)(const craftax_conv_args*);
    int (*scan)(const craftax_scan_args*, void*);
    int (*scan_backward)(const craftax_scan_args*, void*);
    size_t (*scan_saved)(const craftax_scan_args*);
    size_t (*scan_workspace)(const craftax_scan_args*, int);
    int (*norm)(const craftax_norm_args*, void*);
    int (*norm_backward)(const craftax_norm_args*, void*);
    size_t (*norm_workspace)(const craftax_norm_args*);
    int (*recurrence)(const craftax_recurrence_args*, void*);
    int (*recurrence_backward)(const craftax_recurrence_args*, void*);
    size_t (*recurrence_saved)(const craftax_recurrence_args*);
    size_t (*recurrence_workspace)(const craftax_recurrence_args*, int);
    int (*projection)(const craftax_projection_args*, void*);
    int (*projection_backward)(const craftax_projection_args*, void*);
    size_t (*projection_workspace)(const craftax_projection_args*, int);
    int (*dropout)(const craftax_dropout_args*, void*);
    const char* (*last_error)();
} g_lib = {};

template <typename... T> [[noreturn]] void refuse(const T&... parts)
{
    std::ostringstream text;
    (text << ... << parts);
    throw Refusal(text.str());
}

// ---- arguments ------------------------------------------------------------------------------------------
const Tensor* maybe(PyObject* o, const char* name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(name, " must be a tensor");
    return &THPVariable_Unpack(o);
}
const Tensor& need(PyObject* o, const char* name)
{
    const Tensor* t = maybe(o, name);
    if (!t) refuse(name, " is missing");
    return *t;
}

// a dimension, as the C ABI has it
int32_t count(int64_t v, const char* name)
{
    if (v > INT32_MAX) refuse(name, " is beyond 2^31 - 1");
    return (int32_t)v;
}

// an option that is on or off; what has no truth value leaves its own error
bool truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refusal("");
    return v != 0;
}

uint32_t type_code(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return CRAFTAX_F32;
    case at::kBFloat16: return CRAFTAX_BF16;
    case at::kHalf: return CRAFTAX_F16;
    default: refuse("activations must be float32, bfloat16 or float16, not ", t);
    }
}

// What the activations of a call have in common: [steps][n][channels], or [n][channels] for one token.
struct Common {
    at::ScalarType type;
    at::Device device;
    bool token;
    int64_t steps, n, channels;
    explicit Common(const Tensor& x, const char* name) : type(x.scalar_type()), device(x.device())
    {
        if (!x.is_cuda()) refuse("the operators need tensors on a GPU: there is no CPU path");
        if (x.dim() != 2 && x.dim() != 3) refuse(name, " must be [steps][n][channels], or [n][channels] for one token");
        token = x.dim() == 2;
        steps = token ? 1 : x.size(0);
        n = x.size(token ? 0 : 1);
        channels = x.size(token ? 1 : 2);
        if (steps > INT32_MAX || n > INT32_MAX || channels > INT32_MAX) refuse(name, " has a dimension beyond 2^31 - 1");
    }
    at::TensorOptions options(at::ScalarType t) const { return at::TensorOptions().dtype(t).device(device); }
};

void check_kind(const Tensor& t, const char* name, at::ScalarType type, at::Device device)
{
    if (t.scalar_type() != type || t.device() != device) refuse(name, " is ", t.scalar_type(), " on ", t.device(), ", expected ", type, " on ", device);
}

void check_shape(const Tensor& t, const char* name, std::initializer_list<int64_t> shape)
{
    if (t.sizes() != at::IntArrayRef(shape)) refuse(name, " has shape ", t.sizes(), ", expected ", at::IntArrayRef(shape));
}

// [steps][n][inner] or, for one token, [n][inner]
void check_sequence(const Tensor& t, const char* name, const Common& c, int64_t inner)
{
    if (c.token) check_shape(t, name, {c.n, inner});
    else check_shape(t, name, {c.steps, c.n, inner});
}

craftax_view place(const Tensor& t, const Common& c)
{
    return {t.data_ptr(), c.token ? 0 : t.stride(0), t.stride(c.token ? 0 : 1)};
}

// of `channels` values a token
craftax_view sequence_of(const Tensor* t, const char* name, const Common& c, at::ScalarType type, int64_t channels)
{
    if (!t) return {nullptr, 0, 0};
    check_kind(*t, name, type, c.device);
    check_sequence(*t, name, c, channels);
    if (channels != 1 && t->stride(-1) != 1) refuse("the channels of ", name, " must lie side by side");
    return place(*t, c);
}
craftax_view sequence(const Tensor* t, const char* name, const Common& c, at::ScalarType type) { return sequence_of(t, name, c, type, c.channels); }

// b or c, [..][groups][states]; rows that do not lie side by side are copied first (they are short).
craftax_view shared(Tensor& t, const char* name, const Common& c, int64_t groups, int64_t states)
{
    check_kind(t, name, c.type, c.device);
    if (c.token) check_shape(t, name, {c.n, groups, states});
    else check_shape(t, name, {c.steps, c.n, groups, states});
    if ((states != 1 && t.stride(-1) != 1) || (groups != 1 && t.stride(-2) != states)) t = t.contiguous();
    return place(t, c);
}

craftax_view flags(const Tensor* t, const Common& c)
{
    if (!t) return {nullptr, 0, 0};
    if ((t->scalar_type() != at::kByte && t->scalar_type() != at::kBool) || t->device() != c.device) refuse("first must be uint8 or bool on ", c.device);
    if (c.token) check_shape(*t, "first", {c.n});
    else check_shape(*t, "first", {c.steps, c.n});
    return place(*t, c);
}

template <typename T> T* dense(const Tensor* t, const char* name, std::initializer_list<int64_t> shape, at::ScalarType type, const Common& c)
{
    if (!t) return nullptr;
    check_kind(*t, name, type, c.device);
    check_shape(*t, name, shape);
    if (!t->is_contiguous()) refuse(name, " must be contiguous, has strides ", t->strides());
    return static_cast<T*>(t->data_ptr());
}

// ---- outputs ----------------------------------------------------------------------------------------------
// Laid out as t is, the channels side by side.
Tensor like(const Tensor& t)
{
    if (t.is_contiguous()) return at::empty(t.sizes(), t.options());
    Tensor out = at::empty_like(t);
    if (out.stride(-1) != 1) out = at::empty(t.sizes(), t.options());
    return out;
}
// Laid out as b or c, the groups of a token side by side, for sequences as for one token: a view has no stride for them.
Tensor shared_like(const Tensor& t)
{
    Tensor out = like(t);
    if (out.stride(-2) != out.size(-1)) out = at::empty(t.sizes(), t.options());
    return out;
}
// Of `type` and `channels` values a token, steps and environments in the order in which they lie in t.
Tensor like_of(const Tensor& t, const Common& c, at::ScalarType type, int64_t channels)
{
    if (c.token) return at::empty({c.n, channels}, c.options(type));
    if (t.stride(0) < t.stride(1)) return at::empty({c.n, c.steps, channels}, c.options(type)).transpose(0, 1);
    return at::empty({c.steps, c.n, channels}, c.options(type));
}
Tensor like_or_none(const Tensor* t) { return t ? like(*t) : Tensor(); }
void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// A state that the caller gave to be written.  Autograd hears of it as of PyTorch's own operations in place: what kept the state
// for a backward pass refuses to run it, and a state with a history that the write would cut off is not taken.
void check_writable(const Tensor& t)
{
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse("a state that requires gradients cannot be written in place: give out_state, detach the state, or call under torch.no_grad()");
}
void written(const Tensor& t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

Tensor bytes(size_t size, const Common& c) { return size ? at::empty({(int64_t)size}, c.options(at::kByte)) : Tensor(); }

PyObject* wrap(const Tensor& t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* tuple(std::initializer_list<Tensor> values)
{
    PyObject* out = PyTuple_New((Py_ssize_t)values.size());
    Py_ssize_t k = 0;
    for (const Tensor& t : values) {
        PyObject* o = wrap(t);
        if (!o) { Py_DECREF(out); return nullptr; }
        PyTuple_SET_ITEM(out, k++, o);
    }
    return out;
}

template <typename A> void call(int (*entry)(const A*, void*), const A& args, const Common& c)
{
    if (!entry) refuse("the library is not loaded");
    const c10::hip::OptionalHIPGuardMasqueradingAsCUDA guard(c.device);
    const int rc = entry(&args, c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(c.device.index()).stream());
    if (rc != CRAFTAX_OK) refuse(g_lib.last_error(), " (", rc, ")");
}

// ---- the operators: positional arguments, in the order that memory.py gives them -----------------------------
// x, weight, bias, state, first, lengths, silu
craftax_conv_args conv_args(const Common& c, const Tensor& x, PyObject* const* v)
{
    const Tensor& weight = need(v[1], "weight");
    if (weight.dim() != 2) refuse("weight must be [channels][taps]");
    const int64_t taps = weight.size(1);
    craftax_conv_args a = {};
    a.dtype = type_code(c.type);
    a.silu = truth(v[6]);
    a.steps = (int32_t)c.steps; a.n = (int32_t)c.n; a.channels = (int32_t)c.channels; a.taps = count(taps, "taps");
    a.weight = dense<const float>(&weight, "weight", {c.channels, taps}, at::kFloat, c);
    a.bias = dense<const float>(maybe(v[2], "bias"), "bias", {c.channels}, at::kFloat, c);
    a.first = flags(maybe(v[4], "first"), c);
    a.lengths = dense<const int32_t>(maybe(v[5], "lengths"), "lengths", {c.n}, at::kInt, c);
    a.x = sequence(&x, "x", c, c.type);
    a.state_in = dense<const void>(maybe(v[3], "state"), "state", {c.n, taps - 1, c.channels}, c.type, c);
    return a;
}

// .., out_state (None: a new one)
PyObject* causal_conv(PyObject* const* v)
{
    const Tensor& x = need(v[0], "x");
    const Common c(x, "x");
    craftax_conv_args a = conv_args(c, x, v);
    const Tensor y = like(x);
    Tensor out;
    if (const Tensor* given = maybe(v[7], "out_state")) {
        a.state_out = dense<void>(given, "out_state", {c.n, a.taps - 1, c.channels}, c.type, c);
        check_writable(*given);
        out = *given;
    } else {
        out = at::empty({c.n, a.taps < 1 ? 0 : a.taps - 1, c.channels}, c.options(c.type));
        a.state_out = out.data_ptr();
    }
    a.y = place(y, c);
    call(g_lib.conv, a, c);
    if (v[7] != Py_None) written(out);
    return tuple({y, out});
}

// .., dy, dstate
PyObject* causal_conv_backward(PyObject* const* v)
{
    const Tensor &x = need(v[0], "x"), &weight = need(v[1], "weight");
    const Tensor *bias = maybe(v[2], "bias"), *state = maybe(v[3], "state");
    const Common c(x, "x");
    craftax_conv_args a = conv_args(c, x, v);
    const Tensor dx = like(x), dweight = like(weight), dbias = like_or_none(bias), dstate = like_or_none(state);
    a.dy = sequence(&need(v[7], "dy"), "dy", c, c.type);
    a.dx = place(dx, c);
    a.dstate_out = dense<const void>(maybe(v[8], "dstate"), "dstate", {c.n, a.taps - 1, c.channels}, c.type, c);
    a.dstate_in = address(dstate);
    a.dweight = static_cast<float*>(address(dweight));
    a.dbias = static_cast<float*>(address(dbias));
    const Tensor work = bytes(g_lib.conv_workspace ? g_lib.conv_workspace(&a) : 0, c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.conv_backward, a, c);
    return tuple({dx, dweight, dbias, dstate});
}

// x, delta, a, b, c, d, z, delta_bias, softplus, state, first, lengths
craftax_scan_args scan_args(const Common& c, const Tensor& x, PyObject* const* v, Tensor& b, Tensor& cc)
{
    const Tensor& rates = need(v[2], "a");
    b = need(v[3], "b");
    cc = need(v[4], "c");
    if (rates.dim() != 2 || b.dim() != (c.token ? 3 : 4)) refuse("a must be [channels][states], b and c [steps][n][groups][states]");
    const int64_t states = rates.size(1), groups = b.size(-2);
    craftax_scan_args a = {};
    a.dtype = type_code(c.type);
    a.softplus = truth(v[8]);
    a.steps = (int32_t)c.steps; a.n = (int32_t)c.n; a.channels = (int32_t)c.channels;
    a.states = count(states, "states"); a.groups = count(groups, "groups");
    a.a = dense<const float>(&rates, "a", {c.channels, states}, at::kFloat, c);
    a.d = dense<const float>(maybe(v[5], "d"), "d", {c.channels}, at::kFloat, c);
    a.delta_bias = dense<const float>(maybe(v[7], "delta_bias"), "delta_bias", {c.channels}, at::kFloat, c);
    a.first = flags(maybe(v[10], "first"), c);
    a.lengths = dense<const int32_t>(maybe(v[11], "lengths"), "lengths", {c.n}, at::kInt, c);
    a.x = sequence(&x, "x", c, c.type);
    a.delta = sequence(&need(v[1], "delta"), "delta", c, c.type);
    a.z = sequence(maybe(v[6], "z"), "z", c, c.type);
    a.b = shared(b, "b", c, groups, states);
    a.c = shared(cc, "c", c, groups, states);
    a.state_in = dense<const float>(maybe(v[9], "state"), "state", {c.n, c.channels, states}, at::kFloat, c);
    return a;
}

// .., save, out_state (None: a new one)
PyObject* selective_scan(PyObject* const* v)
{
    const Tensor& x = need(v[0], "x");
    const Common c(x, "x");
    Tensor b, cc, out, saved;
    craftax_scan_args a = scan_args(c, x, v, b, cc);
    const Tensor y = like(x);
    if (const Tensor* given = maybe(v[13], "out_state")) {
        a.state_out = dense<float>(given, "out_state", {c.n, c.channels, a.states}, at::kFloat, c);
        check_writable(*given);
        out = *given;
    } else {
        out = at::empty({c.n, c.channels, a.states}, c.options(at::kFloat));
        a.state_out = out.data_ptr<float>();
    }
    a.y = place(y, c);
    if (truth(v[12])) {
        saved = bytes(g_lib.scan_saved ? g_lib.scan_saved(&a) : 0, c);
        a.saved = address(saved);
    }
    const Tensor work = bytes(g_lib.scan_workspace ? g_lib.scan_workspace(&a, 0) : 0, c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.scan, a, c);
    if (v[13] != Py_None) written(out);
    return tuple({y, out, saved});
}

// .., saved, dy, dstate
PyObject* selective_scan_backward(PyObject* const* v)
{
    const Tensor &x = need(v[0], "x"), &delta = need(v[1], "delta"), &rates = need(v[2], "a");
    const Tensor *d = maybe(v[5], "d"), *z = maybe(v[6], "z"), *delta_bias = maybe(v[7], "delta_bias"), *state = maybe(v[9], "state");
    const Tensor* saved = maybe(v[12], "saved");
    const Common c(x, "x");
    Tensor b, cc;
    craftax_scan_args a = scan_args(c, x, v, b, cc);
    if (!saved || saved->scalar_type() != at::kByte || saved->device() != c.device || !saved->is_contiguous() || !g_lib.scan_saved ||
        (size_t)saved->numel() < g_lib.scan_saved(&a))
        refuse("saved is not what selective_scan(..., save=True) returned for these inputs");
    a.saved = saved->data_ptr();
    const Tensor dx = like(x), ddelta = like(delta), da = like(rates), db = shared_like(need(v[3], "b")), dc = shared_like(need(v[4], "c"));
    const Tensor dd = like_or_none(d), dz = like_or_none(z), dbias = like_or_none(delta_bias), dstate = like_or_none(state);
    a.dy = sequence(&need(v[13], "dy"), "dy", c, c.type);
    a.dx = place(dx, c);
    a.ddelta = place(ddelta, c);
    if (dz.defined()) a.dz = place(dz, c);
    a.db = place(db, c);
    a.dc = place(dc, c);
    a.dstate_out = dense<const float>(maybe(v[14], "dstate"), "dstate", {c.n, c.channels, a.states}, at::kFloat, c);
    a.dstate_in = static_cast<float*>(address(dstate));
    a.da = static_cast<float*>(address(da));
    a.dd = static_cast<float*>(address(dd));
    a.ddelta_bias = static_cast<float*>(address(dbias));
    const Tensor work = bytes(g_lib.scan_workspace(&a, 1), c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.scan_backward, a, c);
    return tuple({dx, ddelta, da, db, dc, dd, dz, dbias, dstate});
}

// y, residual, gate, post_weight, scale, pre_weight, gate_act, eps
craftax_norm_args norm_args(const Common& c, const Tensor& y, const Tensor& residual, PyObject* const* v)
{
    if (residual.scalar_type() != c.type && residual.scalar_type() != at::kFloat)
        refuse("residual must be ", c.type, " or float32, not ", residual.scalar_type());
    craftax_norm_args a = {};
    a.dtype = type_code(c.type);
    a.residual_dtype = type_code(residual.scalar_type());
    a.gate_act = (uint32_t)PyLong_AsLong(v[6]);
    a.eps = (float)PyFloat_AsDouble(v[7]);
    if (PyErr_Occurred()) throw Refusal("");
    a.steps = (int32_t)c.steps; a.n = (int32_t)c.n; a.channels = (int32_t)c.channels;
    a.post_weight = dense<const float>(maybe(v[3], "post_weight"), "post_weight", {c.channels}, at::kFloat, c);
    a.scale = dense<const float>(maybe(v[4], "scale"), "scale", {c.channels}, at::kFloat, c);
    a.pre_weight = dense<const float>(maybe(v[5], "pre_weight"), "pre_weight", {c.channels}, at::kFloat, c);
    a.y = sequence(&y, "y", c, c.type);
    a.residual = sequence(&residual, "residual", c, residual.scalar_type());
    a.gate = sequence(maybe(v[2], "gate"), "gate", c, c.type);
    return a;
}

PyObject* residual_norm(PyObject* const* v)
{
    const Tensor &y = need(v[0], "y"), &residual = need(v[1], "residual");
    const Common c(y, "y");
    craftax_norm_args a = norm_args(c, y, residual, v);
    const Tensor out = like(residual), u = like(y);
    a.out = place(out, c);
    a.u = place(u, c);
    call(g_lib.norm, a, c);
    return tuple({out, u});
}

// .., dout, du
PyObject* residual_norm_backward(PyObject* const* v)
{
    const Tensor &y = need(v[0], "y"), &residual = need(v[1], "residual");
    const Tensor* gate = maybe(v[2], "gate");
    const Common c(y, "y");
    craftax_norm_args a = norm_args(c, y, residual, v);
    const Tensor dy = like(y), dresidual = like(residual), dgate = like_or_none(gate);
    const Tensor dpost = like_or_none(maybe(v[3], "post_weight")), dscale = like_or_none(maybe(v[4], "scale")), dpre = like_or_none(maybe(v[5], "pre_weight"));
    a.dout = sequence(maybe(v[8], "dout"), "dout", c, residual.scalar_type());
    a.du = sequence(&need(v[9], "du"), "du", c, c.type);
    a.dy = place(dy, c);
    a.dresidual = place(dresidual, c);
    if (dgate.defined()) a.dgate = place(dgate, c);
    a.dpost_weight = static_cast<float*>(address(dpost));
    a.dscale = static_cast<float*>(address(dscale));
    a.dpre_weight = static_cast<float*>(address(dpre));
    const Tensor work = bytes(g_lib.norm_workspace ? g_lib.norm_workspace(&a) : 0, c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.norm_backward, a, c);
    return tuple({dy, dresidual, dgate, dpost, dscale, dpre});
}

// x, decay, intake, rate, z, state, first, lengths
craftax_recurrence_args recurrence_args(const Common& c, const Tensor& x, PyObject* const* v)
{
    craftax_recurrence_args a = {};
    a.dtype = type_code(c.type);
    a.steps = (int32_t)c.steps; a.n = (int32_t)c.n; a.channels = (int32_t)c.channels;
    a.rate = dense<const float>(&need(v[3], "rate"), "rate", {c.channels}, at::kFloat, c);
    a.first = flags(maybe(v[6], "first"), c);
    a.lengths = dense<const int32_t>(maybe(v[7], "lengths"), "lengths", {c.n}, at::kInt, c);
    a.x = sequence(&x, "x", c, c.type);
    a.decay = sequence(&need(v[1], "decay"), "decay", c, c.type);
    a.intake = sequence(&need(v[2], "intake"), "intake", c, c.type);
    a.z = sequence(maybe(v[4], "z"), "z", c, c.type);
    a.state_in = dense<const float>(maybe(v[5], "state"), "state", {c.n, c.channels}, at::kFloat, c);
    return a;
}

// .., save, out_state (None: a new one)
PyObject* gated_recurrence(PyObject* const* v)
{
    const Tensor& x = need(v[0], "x");
    const Common c(x, "x");
    craftax_recurrence_args a = recurrence_args(c, x, v);
    const Tensor y = like(x);
    Tensor out, saved;
    if (const Tensor* given = maybe(v[9], "out_state")) {
        a.state_out = dense<float>(given, "out_state", {c.n, c.channels}, at::kFloat, c);
        check_writable(*given);
        out = *given;
    } else {
        out = at::empty({c.n, c.channels}, c.options(at::kFloat));
        a.state_out = out.data_ptr<float>();
    }
    a.y = place(y, c);
    if (truth(v[8])) {
        saved = bytes(g_lib.recurrence_saved ? g_lib.recurrence_saved(&a) : 0, c);
        a.saved = address(saved);
    }
    const Tensor work = bytes(g_lib.recurrence_workspace ? g_lib.recurrence_workspace(&a, 0) : 0, c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.recurrence, a, c);
    if (v[9] != Py_None) written(out);
    return tuple({y, out, saved});
}

// .., saved, dy, dstate
PyObject* gated_recurrence_backward(PyObject* const* v)
{
    const Tensor &x = need(v[0], "x"), &decay = need(v[1], "decay"), &intake = need(v[2], "intake"), &rate = need(v[3], "rate");
    const Tensor *z = maybe(v[4], "z"), *state = maybe(v[5], "state"), *saved = maybe(v[8], "saved");
    const Common c(x, "x");
    craftax_recurrence_args a = recurrence_args(c, x, v);
    if (!saved || saved->scalar_type() != at::kByte || saved->device() != c.device || !saved->is_contiguous() || !g_lib.recurrence_saved ||
        (size_t)saved->numel() < g_lib.recurrence_saved(&a))
        refuse("saved is not what gated_recurrence(..., save=True) returned for these inputs");
    a.saved = saved->data_ptr();
    const Tensor dx = like(x), ddecay = like(decay), dintake = like(intake), drate = like(rate), dz = like_or_none(z), dstate = like_or_none(state);
    a.dy = sequence(&need(v[9], "dy"), "dy", c, c.type);
    a.dx = place(dx, c);
    a.ddecay = place(ddecay, c);
    a.dintake = place(dintake, c);
    if (dz.defined()) a.dz = place(dz, c);
    a.dstate_out = dense<const float>(maybe(v[10], "dstate"), "dstate", {c.n, c.channels}, at::kFloat, c);
    a.dstate_in = static_cast<float*>(address(dstate));
    a.drate = static_cast<float*>(address(drate));
    const Tensor work = bytes(g_lib.recurrence_workspace(&a, 1), c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.recurrence_backward, a, c);
    return tuple({dx, ddecay, dintake, drate, dz, dstate});
}

// x, weight, bias, act
craftax_projection_args projection_args(const Common& c, const Tensor& x, PyObject* const* v)
{
    const Tensor& weight = need(v[1], "weight");
    if (weight.dim() != 2) refuse("weight must be [outputs][inputs]");
    check_kind(weight, "weight", c.type, c.device);
    check_shape(weight, "weight", {weight.size(0), c.channels});
    craftax_projection_args a = {};
    a.dtype = type_code(c.type);
    a.act = (uint32_t)PyLong_AsLong(v[3]);
    if (PyErr_Occurred()) throw Refusal("");
    a.steps = (int32_t)c.steps; a.n = (int32_t)c.n; a.inputs = (int32_t)c.channels; a.outputs = count(weight.size(0), "outputs");
    a.weight = weight.data_ptr();
    a.weight_row = weight.stride(0); a.weight_column = weight.stride(1);
    if (a.weight_row != 1 && a.weight_column != 1 && a.inputs > 1 && a.outputs > 1) refuse("the inputs or the outputs of weight must lie side by side");
    a.bias = dense<const float>(maybe(v[2], "bias"), "bias", {a.outputs}, at::kFloat, c);
    a.x = sequence(&x, "x", c, c.type);
    return a;
}

// the type of a tensor of outputs, which is the activations' or float32
at::ScalarType wide_type(const Tensor& t, const char* name, const Common& c)
{
    if (t.scalar_type() != c.type && t.scalar_type() != at::kFloat) refuse(name, " must be ", c.type, " or float32, not ", t.scalar_type());
    return t.scalar_type();
}

// .., residual, save
PyObject* projection(PyObject* const* v)
{
    const Tensor& x = need(v[0], "x");
    const Tensor* residual = maybe(v[4], "residual");
    const Common c(x, "x");
    craftax_projection_args a = projection_args(c, x, v);
    const at::ScalarType type = residual ? wide_type(*residual, "residual", c) : c.type;
    a.out_dtype = type_code(type);
    a.residual = sequence_of(residual, "residual", c, type, a.outputs);
    const Tensor out = like_of(x, c, type, a.outputs);
    Tensor pre;
    a.out = place(out, c);
    if (truth(v[5])) {
        pre = like_of(x, c, c.type, a.outputs);
        a.pre = place(pre, c);
    }
    const Tensor work = bytes(g_lib.projection_workspace ? g_lib.projection_workspace(&a, 0) : 0, c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.projection, a, c);
    return tuple({out, pre});
}

// .., pre, dout, whether the gradients of x and of weight are wanted, and whether the latter is float32
PyObject* projection_backward(PyObject* const* v)
{
    const Tensor& x = need(v[0], "x");
    const Tensor *bias = maybe(v[2], "bias"), *pre = maybe(v[4], "pre");
    const Tensor& dout = need(v[5], "dout");
    const Common c(x, "x");
    craftax_projection_args a = projection_args(c, x, v);
    const at::ScalarType type = wide_type(dout, "dout", c);
    a.out_dtype = type_code(type);
    a.dout = sequence_of(&dout, "dout", c, type, a.outputs);
    a.pre = sequence_of(pre, "pre", c, c.type, a.outputs);
    Tensor dx, dweight, dbias = like_or_none(bias);
    if (truth(v[6])) {
        dx = like(x);
        a.dx = place(dx, c);
    }
    a.dweight_dtype = a.dtype;
    if (truth(v[7])) {
        const at::ScalarType kept = truth(v[8]) ? at::kFloat : c.type;
        dweight = at::empty({a.outputs, c.channels}, c.options(kept));
        a.dweight = dweight.data_ptr();
        a.dweight_dtype = type_code(kept);
    }
    a.dbias = static_cast<float*>(address(dbias));
    const Tensor work = bytes(g_lib.projection_workspace ? g_lib.projection_workspace(&a, 1) : 0, c);
    a.workspace = address(work);
    a.workspace_bytes = work.defined() ? (size_t)work.numel() : 0;
    call(g_lib.projection_backward, a, c);
    return tuple({dx, dweight, dbias});
}

int64_t whole(PyObject* o, const char* name)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(name, " must be a whole number below 2^63");
    }
    return v;
}

// x, residual, p, seed, step, step_at, env, type of the output (a code; below 0: as residual or x)
PyObject* residual_dropout(PyObject* const* v)
{
    const Tensor& x = need(v[0], "x");
    const Tensor *residual = maybe(v[1], "residual"), *step_at = maybe(v[5], "step");
    const Common c(x, "x");
    craftax_dropout_args a = {};
    a.dtype = type_code(c.type);
    a.steps = (int32_t)c.steps; a.n = (int32_t)c.n; a.channels = (int32_t)c.channels;
    a.p = PyFloat_AsDouble(v[2]);
    if (PyErr_Occurred()) throw Refusal("");
    a.seed = PyLong_AsUnsignedLongLong(v[3]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        refuse("seed must be a whole number of 0..2^64 - 1");
    }
    a.step = whole(v[4], "step"); a.env = whole(v[6], "env");
    if (step_at) {
        check_kind(*step_at, "step", at::kLong, c.device);
        if (step_at->numel() != 1) refuse("step must be one number");
        a.step_at = step_at->data_ptr<int64_t>();
    }
    const int64_t code = whole(v[7], "dtype");
    at::ScalarType type = residual ? wide_type(*residual, "residual", c) : c.type;
    if (code >= 0) type = code == CRAFTAX_F32 ? at::kFloat : code == CRAFTAX_BF16 ? at::kBFloat16 : at::kHalf;
    a.out_dtype = type_code(type);
    a.x = sequence(&x, "x", c, c.type);
    a.residual = sequence(residual, "residual", c, type);
    const Tensor out = type == c.type ? like(x) : like_of(x, c, type, c.channels);
    a.out = place(out, c);
    call(g_lib.dropout, a, c);
    return wrap(out);
}

// ---- module -----------------------------------------------------------------------------------------------
template <PyObject* (*F)(PyObject* const*), int COUNT>
PyObject* entry(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    if (count != COUNT) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", COUNT, count);
        return nullptr;
    }
    try {
        return F(v);
    } catch (const Refusal& e) {
        if (!PyErr_Occurred()) PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, e.what());
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(g_no_memory ? g_no_memory : PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// bind(error class, class of errors for want of memory, addresses of the entry points in the order of Library)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t count)
{
    constexpr Py_ssize_t ENTRIES = sizeof(Library) / sizeof(void*);
    if (count != 2 + ENTRIES) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", 2 + ENTRIES, count);
        return nullptr;
    }
    void* at[ENTRIES];
    for (Py_ssize_t k = 0; k < ENTRIES; ++k) {
        at[k] = PyLong_AsVoidPtr(v[2 + k]);
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof(at) == sizeof(Library), "one address per entry point");
    std::memcpy(&g_lib, at, sizeof(at));
    Py_INCREF(v[0]);
    Py_XDECREF(g_error);
    g_error = v[0];
    Py_INCREF(v[1]);
    Py_XDECREF(g_no_memory);
    g_no_memory = v[1];
    Py_RETURN_NONE;
}

#define CRAFTAX_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f))
PyMethodDef g_methods[] = {
    {"bind", CRAFTAX_FAST(&bind), METH_FASTCALL, nullptr},
    {"causal_conv", CRAFTAX_FAST((&entry<causal_conv, 8>)), METH_FASTCALL, nullptr},
    {"causal_conv_backward", CRAFTAX_FAST((&entry<causal_conv_backward, 9>)), METH_FASTCALL, nullptr},
    {"selective_scan", CRAFTAX_FAST((&entry<selective_scan, 14>)), METH_FASTCALL, nullptr},
    {"selective_scan_backward", CRAFTAX_FAST((&entry<selective_scan_backward, 15>)), METH_FASTCALL, nullptr},
    {"residual_norm", CRAFTAX_FAST((&entry<residual_norm, 8>)), METH_FASTCALL, nullptr},
    {"residual_norm_backward", CRAFTAX_FAST((&entry<residual_norm_backward, 10>)), METH_FASTCALL, nullptr},
    {"gated_recurrence", CRAFTAX_FAST((&entry<gated_recurrence, 10>)), METH_FASTCALL, nullptr},
    {"gated_recurrence_backward", CRAFTAX_FAST((&entry<gated_recurrence_backward, 11>)), METH_FASTCALL, nullptr},
    {"projection", CRAFTAX_FAST((&entry<projection, 6>)), METH_FASTCALL, nullptr},
    {"projection_backward", CRAFTAX_FAST((&entry<projection_backward, 9>)), METH_FASTCALL, nullptr},
    {"residual_dropout", CRAFTAX_FAST((&entry<residual_dropout, 8>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&g_module); }
