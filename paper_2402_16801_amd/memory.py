"""Operators of a policy with memory on PyTorch tensors (see include/craftax.h for what they compute).

A policy sees a small window of its world, so it carries a memory from step to step.  These are the
parts of a recurrent policy block that are no plain matrix product:

  causal_conv, causal_conv_backward, causal_conv_step              short causal convolution per channel
  selective_scan, selective_scan_backward, selective_scan_step     selective state space scan
  residual_norm, residual_norm_backward                            norm, gate, scale, residual, norm

Sequences are [steps][n][channels], the order of rollouts; a batch-first tensor is passed as its
`.transpose(0, 1)` (any strides of the first two dimensions are taken, the channels lie side by
side).  `first` (uint8 or bool [steps][n]) marks steps at which an episode begins, as the simulator's
`done` does for the observation that came with it; `lengths` (int32 [n]) says how many steps of each
environment count.  The `*_step` forms take one token, [n][channels], and update the state in place
unless `out_state` is given.  Activations are float32, bfloat16 or float16, parameters and the states
of the scan float32; a convolution's state has the type of its input.

Argument marshalling only: outputs and workspaces are allocated here, the work runs in the HIP
kernels, on the current stream of the tensors' device.  `conv`, `scan` and `norm` are the same
operators as differentiable functions.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding
from .binding import ConvArgs, CraftaxError, NormArgs, ScanArgs

Tensor = torch.Tensor
_DTYPES = {torch.float32: binding.F32, torch.bfloat16: binding.BF16, torch.float16: binding.F16}
_GATES = {"sigmoid": binding.GATE_SIGMOID, "silu": binding.GATE_SILU, "linear": binding.GATE_LINEAR}
_NONE = (None, 0, 0)


class ConvGrads(NamedTuple):
    x: Tensor
    weight: Tensor
    bias: Optional[Tensor]
    state: Optional[Tensor]


class ScanGrads(NamedTuple):
    x: Tensor
    delta: Tensor
    a: Tensor
    b: Tensor
    c: Tensor
    d: Optional[Tensor]
    z: Optional[Tensor]
    delta_bias: Optional[Tensor]
    state: Optional[Tensor]


class NormGrads(NamedTuple):
    y: Tensor
    residual: Tensor
    gate: Optional[Tensor]
    post_weight: Optional[Tensor]
    scale: Optional[Tensor]
    pre_weight: Optional[Tensor]


# ---- checks ------------------------------------------------------------------------------------------

def _refuse(text):
    raise CraftaxError(text)


def _dtype(x):
    if not x.is_cuda:
        _refuse("the operators need tensors on a GPU: there is no CPU path")
    code = _DTYPES.get(x.dtype)
    if code is None:
        _refuse(f"activations must be float32, bfloat16 or float16, not {x.dtype}")
    return code


def _seq(name, v, shape, dtype, device):
    """(address, stride of steps, stride of environments) of a sequence or, with two dimensions, of one token."""
    if v is None:
        return _NONE
    if v.dtype != dtype or v.device != device:
        _refuse(f"{name} is {v.dtype} on {v.device}, expected {dtype} on {device}")
    if v.shape != shape:
        _refuse(f"{name} has shape {tuple(v.shape)}, expected {tuple(shape)}")
    strides = v.stride()
    if strides[-1] != 1 and shape[-1] != 1:
        _refuse(f"the channels of {name} must lie side by side")
    return (v.data_ptr(), strides[0], strides[1]) if len(shape) >= 3 else (v.data_ptr(), 0, strides[0])


def _shared(name, v, token, groups, states, dtype, device):
    """b or c, [..][groups][states].  Rows are read by whole words: others are copied first (they are
    short: states values against channels)."""
    shape = token[:-1] + (groups, states)
    if v.shape != shape:
        _refuse(f"{name} has shape {tuple(v.shape)}, expected {tuple(shape)}")
    if v.dtype != dtype or v.device != device:
        _refuse(f"{name} is {v.dtype} on {v.device}, expected {dtype} on {device}")
    strides, size = v.stride(), v.element_size()
    if strides[-1] != 1 or (groups > 1 and strides[-2] != states) or v.data_ptr() % 4 or any(s * size % 4 for s in strides[:-2]):
        v = v.contiguous()
        if v.data_ptr() % 4:
            v = v.clone()
        strides = v.stride()
    return v, (v.data_ptr(), strides[0], strides[1]) if len(shape) == 4 else (v.data_ptr(), 0, strides[0])


def _flags(first, shape, device):
    if first is None:
        return _NONE
    if first.dtype not in (torch.uint8, torch.bool) or first.device != device:
        _refuse(f"first must be uint8 or bool on {device}")
    if first.shape != shape:
        _refuse(f"first has shape {tuple(first.shape)}, expected {tuple(shape)}")
    strides = first.stride()
    return (first.data_ptr(), strides[0], strides[1]) if len(shape) == 2 else (first.data_ptr(), 0, strides[0])


def _dense(name, v, shape, dtype, device):
    """Address of a contiguous tensor, None for None."""
    if v is None:
        return None
    if v.dtype != dtype or v.device != device:
        _refuse(f"{name} is {v.dtype} on {v.device}, expected {dtype} on {device}")
    if v.shape != shape or not v.is_contiguous():
        _refuse(f"{name} must be contiguous of shape {tuple(shape)}, is {tuple(v.shape)} with strides {v.stride()}")
    return v.data_ptr()


def _like(v, dtype=None):
    """An output laid out as v is, its last dimension side by side."""
    out = torch.empty_like(v, dtype=dtype)
    if out.stride(-1) != 1 or (out.dim() == 4 and out.stride(-2) != out.shape[-1]):
        out = torch.empty(v.shape, dtype=dtype or v.dtype, device=v.device)
    return out


def _ptr(v):
    return None if v is None else v.data_ptr()


def _place(v):
    return _NONE if v is None else (v.data_ptr(), v.stride(0), v.stride(1))


def _call(name, args, device):
    lib = binding.load()
    stream = torch.cuda.current_stream(device).cuda_stream
    if device.index == torch.cuda.current_device():
        rc = getattr(lib, name)(args, stream)
    else:
        with torch.cuda.device(device):
            rc = getattr(lib, name)(args, stream)
    if rc != 0:
        binding._check(rc, name)


def _work(args, size, device):
    """Gives the call its workspace; the tensor has to live until the call is enqueued."""
    if size == 0:
        return None
    work = torch.empty(size, dtype=torch.uint8, device=device)
    args.workspace, args.workspace_bytes = work.data_ptr(), size
    return work


# ---- short causal convolution ---------------------------------------------------------------------------

def _conv_args(x, weight, bias, state, first, lengths, silu):
    code, device, shape = _dtype(x), x.device, x.shape
    if len(shape) not in (2, 3):
        _refuse("x must be [steps][n][channels], or [n][channels] for one token")
    steps, n, channels = shape if len(shape) == 3 else (1, *shape)
    taps = weight.shape[-1]
    f32 = torch.float32
    return ConvArgs(code, int(silu), steps, n, channels, taps, _dense("weight", weight, (channels, taps), f32, device),
                    _dense("bias", bias, (channels,), f32, device), *_flags(first, shape[:-1], device),
                    _dense("lengths", lengths, (n,), torch.int32, device), *_seq("x", x, shape, x.dtype, device), *_NONE,
                    _dense("state", state, (n, taps - 1, channels), x.dtype, device))


def causal_conv(x, weight, bias=None, *, state=None, first=None, lengths=None, silu=True):
    """(y, state after the last step).  weight: [channels][taps], the newest input last."""
    args = _conv_args(x, weight, bias, state, first, lengths, silu)
    y = _like(x)
    out = torch.empty((args.n, args.taps - 1, args.channels), dtype=x.dtype, device=x.device)
    args.y, args.y_step, args.y_env = _place(y)
    args.state_out = out.data_ptr()
    _call("craftax_causal_conv", args, x.device)
    return y, out


def causal_conv_backward(dy, x, weight, bias=None, *, state=None, first=None, lengths=None, silu=True, dstate=None) -> ConvGrads:
    """Gradients for dy = dL/dy and dstate = dL/d(state after the last step); the rest as in the forward call."""
    args = _conv_args(x, weight, bias, state, first, lengths, silu)
    device = x.device
    dx, dweight = _like(x), torch.empty_like(weight)
    dbias = None if bias is None else torch.empty_like(bias)
    dstate_in = None if state is None else torch.empty_like(state)
    args.dy, args.dy_step, args.dy_env = _seq("dy", dy, x.shape, x.dtype, device)
    args.dx, args.dx_step, args.dx_env = _place(dx)
    args.dstate_out = _dense("dstate", dstate, (args.n, args.taps - 1, args.channels), x.dtype, device)
    args.dstate_in, args.dweight, args.dbias = _ptr(dstate_in), dweight.data_ptr(), _ptr(dbias)
    work = _work(args, binding.load().craftax_causal_conv_workspace_bytes(args), device)
    _call("craftax_causal_conv_backward", args, device)
    del work
    return ConvGrads(dx, dweight, dbias, dstate_in)


def causal_conv_step(x, weight, bias, state, *, first=None, silu=True, out_state=None):
    """One token: (y, state).  The state is updated in place unless out_state is given."""
    args = _conv_args(x, weight, bias, state, first, None, silu)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    out = state if out_state is None else out_state
    args.y, args.y_env = y.data_ptr(), args.channels
    args.state_out = _dense("out_state", out, (args.n, args.taps - 1, args.channels), x.dtype, x.device)
    _call("craftax_causal_conv", args, x.device)
    return y, out


# ---- selective state space scan ---------------------------------------------------------------------------

def _scan_args(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, lengths):
    """(arguments, b, c): b and c are returned because they may be copies."""
    code, device, shape, dtype = _dtype(x), x.device, x.shape, x.dtype
    if len(shape) not in (2, 3):
        _refuse("x must be [steps][n][channels], or [n][channels] for one token")
    if b.dim() != len(shape) + 1 or a.dim() != 2:
        _refuse("a must be [channels][states], b and c [steps][n][groups][states]")
    steps, n, channels = shape if len(shape) == 3 else (1, *shape)
    states, groups = a.shape[1], b.shape[-2]
    f32 = torch.float32
    b, b_place = _shared("b", b, shape, groups, states, dtype, device)
    c, c_place = _shared("c", c, shape, groups, states, dtype, device)
    args = ScanArgs(code, int(softplus), steps, n, channels, states, groups, _dense("a", a, (channels, states), f32, device),
                    _dense("d", d, (channels,), f32, device), _dense("delta_bias", delta_bias, (channels,), f32, device),
                    *_flags(first, shape[:-1], device), _dense("lengths", lengths, (n,), torch.int32, device),
                    *_seq("x", x, shape, dtype, device), *_seq("delta", delta, shape, dtype, device), *_seq("z", z, shape, dtype, device), *_NONE,
                    *b_place, *c_place, _dense("state", state, (n, channels, states), f32, device))
    return args, b, c


def selective_scan(x, delta, a, b, c, *, d=None, z=None, delta_bias=None, softplus=True, state=None, first=None, lengths=None, save=False):
    """(y, state after the last step, saved).  saved is what a backward pass needs, None without `save`."""
    args, b, c = _scan_args(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, lengths)
    device, lib = x.device, binding.load()
    y = _like(x)
    out = torch.empty((args.n, args.channels, args.states), dtype=torch.float32, device=device)
    saved = None
    if save:
        saved = torch.empty(lib.craftax_selective_scan_saved_bytes(args), dtype=torch.uint8, device=device)
        args.saved = saved.data_ptr()
    args.y, args.y_step, args.y_env = _place(y)
    args.state_out = out.data_ptr()
    work = _work(args, lib.craftax_selective_scan_workspace_bytes(args, 0), device)
    _call("craftax_selective_scan", args, device)
    del work
    return y, out, saved


def selective_scan_backward(dy, saved, x, delta, a, b, c, *, d=None, z=None, delta_bias=None, softplus=True, state=None, first=None, lengths=None,
                            dstate=None) -> ScanGrads:
    """Gradients for dy = dL/dy and dstate = dL/d(state after the last step); `saved` from the forward call, the
    rest as it was there."""
    given_b, given_c = b, c
    args, b, c = _scan_args(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, lengths)
    device, lib = x.device, binding.load()
    if saved is None or saved.numel() * saved.element_size() < lib.craftax_selective_scan_saved_bytes(args):
        _refuse("saved is not what selective_scan(..., save=True) returned for these inputs")
    args.saved = _dense("saved", saved, saved.shape, torch.uint8, device)
    dx, ddelta, db, dc = _like(x), _like(delta), _like(given_b), _like(given_c)
    dz = None if z is None else _like(z)
    da = torch.empty_like(a)
    dd = None if d is None else torch.empty_like(d)
    dbias = None if delta_bias is None else torch.empty_like(delta_bias)
    dstate_in = None if state is None else torch.empty_like(state)
    args.dy, args.dy_step, args.dy_env = _seq("dy", dy, x.shape, x.dtype, device)
    args.dx, args.dx_step, args.dx_env = _place(dx)
    args.ddelta, args.ddelta_step, args.ddelta_env = _place(ddelta)
    args.dz, args.dz_step, args.dz_env = _place(dz)
    args.db, args.db_step, args.db_env = _place(db)
    args.dc, args.dc_step, args.dc_env = _place(dc)
    args.dstate_out = _dense("dstate", dstate, (args.n, args.channels, args.states), torch.float32, device)
    args.dstate_in, args.da, args.dd, args.ddelta_bias = _ptr(dstate_in), da.data_ptr(), _ptr(dd), _ptr(dbias)
    work = _work(args, lib.craftax_selective_scan_workspace_bytes(args, 1), device)
    _call("craftax_selective_scan_backward", args, device)
    del work
    return ScanGrads(dx, ddelta, da, db, dc, dd, dz, dbias, dstate_in)


def selective_scan_step(x, delta, a, b, c, state, *, d=None, z=None, delta_bias=None, softplus=True, first=None, out_state=None):
    """One token: (y, state); b and c are [n][groups][states].  The state is updated in place unless out_state is given."""
    args, b, c = _scan_args(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, None)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    out = state if out_state is None else out_state
    args.y, args.y_env = y.data_ptr(), args.channels
    args.state_out = _dense("out_state", out, (args.n, args.channels, args.states), torch.float32, x.device)
    _call("craftax_selective_scan", args, x.device)
    return y, out


# ---- norm, gate, scale, residual, norm ----------------------------------------------------------------------

def _norm_args(y, residual, gate, post_weight, scale, pre_weight, gate_act, eps):
    code, device, shape, f32 = _dtype(y), y.device, y.shape, torch.float32
    if len(shape) not in (2, 3):
        _refuse("y must be [steps][n][channels], or [rows][channels]")
    if gate_act not in _GATES:
        _refuse(f"gate_act must be one of {sorted(_GATES)}")
    if residual.dtype not in (y.dtype, f32):
        _refuse(f"residual must be {y.dtype} or float32, not {residual.dtype}")
    steps, n, channels = shape if len(shape) == 3 else (1, *shape)
    return NormArgs(code, _DTYPES[residual.dtype], _GATES[gate_act], steps, n, channels, eps,
                    _dense("post_weight", post_weight, (channels,), f32, device), _dense("scale", scale, (channels,), f32, device),
                    _dense("pre_weight", pre_weight, (channels,), f32, device), *_seq("y", y, shape, y.dtype, device),
                    *_seq("residual", residual, shape, residual.dtype, device), *_seq("gate", gate, shape, y.dtype, device))


def _rows(v):
    return _place(v) if v is None or v.dim() == 3 else (v.data_ptr(), 0, v.stride(0))


def residual_norm(y, residual, *, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid", eps=1e-6):
    """(out, u): out = residual + norm(y) * scale * act(gate), u = norm(out)."""
    args = _norm_args(y, residual, gate, post_weight, scale, pre_weight, gate_act, eps)
    out, u = _like(residual), _like(y)
    args.out, args.out_step, args.out_env = _rows(out)
    args.u, args.u_step, args.u_env = _rows(u)
    _call("craftax_residual_norm", args, y.device)
    return out, u


def residual_norm_backward(dout, du, y, residual, *, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid",
                           eps=1e-6) -> NormGrads:
    """Gradients for dout = dL/d(out), which may be None, and du = dL/du; the rest as in the forward call."""
    args = _norm_args(y, residual, gate, post_weight, scale, pre_weight, gate_act, eps)
    device = y.device
    dy, dresidual = _like(y), _like(residual)
    dgate = None if gate is None else _like(gate)
    weights = [None if v is None else torch.empty_like(v) for v in (post_weight, scale, pre_weight)]
    args.dout, args.dout_step, args.dout_env = _seq("dout", dout, y.shape, residual.dtype, device)
    args.du, args.du_step, args.du_env = _seq("du", du, y.shape, y.dtype, device)
    args.dy, args.dy_step, args.dy_env = _rows(dy)
    args.dresidual, args.dresidual_step, args.dresidual_env = _rows(dresidual)
    if dgate is not None:
        args.dgate, args.dgate_step, args.dgate_env = _rows(dgate)
    args.dpost_weight, args.dscale, args.dpre_weight = (_ptr(v) for v in weights)
    work = _work(args, binding.load().craftax_residual_norm_workspace_bytes(args), device)
    _call("craftax_residual_norm_backward", args, device)
    del work
    return NormGrads(dy, dresidual, dgate, *weights)


# ---- the same as differentiable functions ---------------------------------------------------------------------

def _side_by_side(g, like):
    """A gradient as autograd hands it over: expanded or transposed ones are made dense."""
    if g is None:
        return None
    g = g.to(like.dtype)
    return g if g.stride(-1) == 1 else g.contiguous()


class _Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, first, lengths, silu):
        y, out = causal_conv(x, weight, bias, state=state, first=first, lengths=lengths, silu=silu)
        ctx.save_for_backward(x, weight, bias, state, first, lengths)
        ctx.silu = silu
        return y, out

    @staticmethod
    def backward(ctx, dy, dstate):
        x, weight, bias, state, first, lengths = ctx.saved_tensors
        g = causal_conv_backward(_side_by_side(dy, x), x, weight, bias, state=state, first=first, lengths=lengths, silu=ctx.silu,
                                 dstate=dstate.contiguous())
        return g.x, g.weight, g.bias, g.state, None, None, None


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, delta, a, b, c, d, z, delta_bias, state, first, lengths, softplus):
        y, out, saved = selective_scan(x, delta, a, b, c, d=d, z=z, delta_bias=delta_bias, softplus=softplus, state=state, first=first,
                                       lengths=lengths, save=True)
        ctx.save_for_backward(saved, x, delta, a, b, c, d, z, delta_bias, state, first, lengths)
        ctx.softplus = softplus
        return y, out

    @staticmethod
    def backward(ctx, dy, dstate):
        saved, x, delta, a, b, c, d, z, delta_bias, state, first, lengths = ctx.saved_tensors
        g = selective_scan_backward(_side_by_side(dy, x), saved, x, delta, a, b, c, d=d, z=z, delta_bias=delta_bias, softplus=ctx.softplus,
                                    state=state, first=first, lengths=lengths, dstate=dstate.contiguous())
        return g.x, g.delta, g.a, g.b, g.c, g.d, g.z, g.delta_bias, g.state, None, None, None


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, residual, gate, post_weight, scale, pre_weight, gate_act, eps):
        ctx.save_for_backward(y, residual, gate, post_weight, scale, pre_weight)
        ctx.how = {"gate_act": gate_act, "eps": eps}
        return residual_norm(y, residual, gate=gate, post_weight=post_weight, scale=scale, pre_weight=pre_weight, **ctx.how)

    @staticmethod
    def backward(ctx, dout, du):
        y, residual, gate, post_weight, scale, pre_weight = ctx.saved_tensors
        g = residual_norm_backward(_side_by_side(dout, residual), _side_by_side(du, y), y, residual, gate=gate, post_weight=post_weight,
                                   scale=scale, pre_weight=pre_weight, **ctx.how)
        return g.y, g.residual, g.gate, g.post_weight, g.scale, g.pre_weight, None, None


def conv(x, weight, bias=None, *, state=None, first=None, lengths=None, silu=True):
    """causal_conv, differentiable in x, weight, bias and state."""
    return _Conv.apply(x, weight, bias, state, first, lengths, silu)


def scan(x, delta, a, b, c, *, d=None, z=None, delta_bias=None, softplus=True, state=None, first=None, lengths=None):
    """selective_scan, differentiable in every tensor but first and lengths: (y, state after the last step)."""
    return _Scan.apply(x, delta, a, b, c, d, z, delta_bias, state, first, lengths, softplus)


def norm(y, residual, *, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid", eps=1e-6):
    """residual_norm, differentiable in every tensor."""
    return _Norm.apply(y, residual, gate, post_weight, scale, pre_weight, gate_act, eps)
