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
unless `out_state` is given; as with PyTorch's operations in place, a state that requires gradients is
refused there, and a backward pass that needs the state as it was raises.  Activations are float32,
bfloat16 or float16, parameters and the states of the scan float32; a convolution's state has the type
of its input.

Argument marshalling only (in csrc/marshal.cpp): outputs and workspaces are allocated, the work runs
in the HIP kernels, on the current stream of the tensors' device.  `conv`, `scan` and `norm` are the
same operators as functions that can be differentiated once.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding
from .binding import CraftaxError

try:
    from . import _marshal
except ImportError as e:
    raise CraftaxError(f"paper_2402_16801_amd/_marshal.so is missing or does not load ({e}): build it first "
                       "(python -c 'import __graft_entry__ as g; g.build()')") from e

Tensor = torch.Tensor
_GATES = {"sigmoid": binding.GATE_SIGMOID, "silu": binding.GATE_SILU, "linear": binding.GATE_LINEAR}
_ENTRIES = ("causal_conv", "causal_conv_backward", "causal_conv_workspace_bytes", "selective_scan", "selective_scan_backward",
            "selective_scan_saved_bytes", "selective_scan_workspace_bytes", "residual_norm", "residual_norm_backward",
            "residual_norm_workspace_bytes", "last_error")
_bound = None


def _ready():
    """The marshalling module, with the entry points of the library that binding has loaded."""
    global _bound
    if _bound is None or _bound is not binding._lib:
        lib = binding.load()
        _marshal.bind(CraftaxError, torch.OutOfMemoryError, *(ctypes.cast(getattr(lib, "craftax_" + name), ctypes.c_void_p).value for name in _ENTRIES))
        _bound = lib
    return _marshal


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


# ---- short causal convolution ---------------------------------------------------------------------------

def causal_conv(x, weight, bias=None, *, state=None, first=None, lengths=None, silu=True):
    """(y, state after the last step).  weight: [channels][taps], the newest input last."""
    return _ready().causal_conv(x, weight, bias, state, first, lengths, silu, None)


def causal_conv_backward(dy, x, weight, bias=None, *, state=None, first=None, lengths=None, silu=True, dstate=None) -> ConvGrads:
    """Gradients for dy = dL/dy and dstate = dL/d(state after the last step); the rest as in the forward call."""
    return ConvGrads._make(_ready().causal_conv_backward(x, weight, bias, state, first, lengths, silu, dy, dstate))


def causal_conv_step(x, weight, bias, state, *, first=None, silu=True, out_state=None):
    """One token: (y, state).  The state is updated in place unless out_state is given."""
    return _ready().causal_conv(x, weight, bias, state, first, None, silu, state if out_state is None else out_state)


# ---- selective state space scan ---------------------------------------------------------------------------

def selective_scan(x, delta, a, b, c, *, d=None, z=None, delta_bias=None, softplus=True, state=None, first=None, lengths=None, save=False):
    """(y, state after the last step, saved).  saved is what a backward pass needs, None without `save`."""
    return _ready().selective_scan(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, lengths, save, None)


def selective_scan_backward(dy, saved, x, delta, a, b, c, *, d=None, z=None, delta_bias=None, softplus=True, state=None, first=None, lengths=None,
                            dstate=None) -> ScanGrads:
    """Gradients for dy = dL/dy and dstate = dL/d(state after the last step); `saved` from the forward call, the
    rest as it was there."""
    return ScanGrads._make(_ready().selective_scan_backward(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, lengths, saved, dy, dstate))


def selective_scan_step(x, delta, a, b, c, state, *, d=None, z=None, delta_bias=None, softplus=True, first=None, out_state=None):
    """One token: (y, state); b and c are [n][groups][states].  The state is updated in place unless out_state is given."""
    return _ready().selective_scan(x, delta, a, b, c, d, z, delta_bias, softplus, state, first, None, False,
                                   state if out_state is None else out_state)[:2]


# ---- norm, gate, scale, residual, norm ----------------------------------------------------------------------

def _gate_act(name):
    if name not in _GATES:
        raise CraftaxError(f"gate_act must be one of {sorted(_GATES)}")
    return _GATES[name]


def residual_norm(y, residual, *, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid", eps=1e-6):
    """(out, u): out = residual + norm(y) * scale * act(gate), u = norm(out)."""
    return _ready().residual_norm(y, residual, gate, post_weight, scale, pre_weight, _gate_act(gate_act), eps)


def residual_norm_backward(dout, du, y, residual, *, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid",
                           eps=1e-6) -> NormGrads:
    """Gradients for dout = dL/d(out), which may be None, and du = dL/du; the rest as in the forward call."""
    return NormGrads._make(_ready().residual_norm_backward(y, residual, gate, post_weight, scale, pre_weight, _gate_act(gate_act), eps, dout, du))


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
    @once_differentiable
    def backward(ctx, dy, dstate):
        x, weight, bias, state, first, lengths = ctx.saved_tensors
        g = causal_conv_backward(_side_by_side(dy, x), x, weight, bias, state=state, first=first, lengths=lengths, silu=ctx.silu,
                                 dstate=dstate.contiguous())
        return g.x, g.weight, g.bias, g.state, None, None, None


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, delta, a, b, c, d, z, delta_bias, state, first, lengths, softplus, save):
        y, out, saved = selective_scan(x, delta, a, b, c, d=d, z=z, delta_bias=delta_bias, softplus=softplus, state=state, first=first,
                                       lengths=lengths, save=save)
        ctx.save_for_backward(saved, x, delta, a, b, c, d, z, delta_bias, first, lengths)
        # not among the saved tensors: its values are in `saved`, so that it may be written before the backward pass
        ctx.state = None if state is None else state.detach()
        ctx.softplus = softplus
        return y, out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dstate):
        saved, x, delta, a, b, c, d, z, delta_bias, first, lengths = ctx.saved_tensors
        g = selective_scan_backward(_side_by_side(dy, x), saved, x, delta, a, b, c, d=d, z=z, delta_bias=delta_bias, softplus=ctx.softplus,
                                    state=ctx.state, first=first, lengths=lengths, dstate=dstate.contiguous())
        return g.x, g.delta, g.a, g.b, g.c, g.d, g.z, g.delta_bias, g.state, None, None, None, None


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, residual, gate, post_weight, scale, pre_weight, gate_act, eps):
        ctx.save_for_backward(y, residual, gate, post_weight, scale, pre_weight)
        ctx.how = {"gate_act": gate_act, "eps": eps}
        return residual_norm(y, residual, gate=gate, post_weight=post_weight, scale=scale, pre_weight=pre_weight, **ctx.how)

    @staticmethod
    @once_differentiable
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
    # what a backward pass needs is kept only where one can follow
    save = torch.is_grad_enabled() and any(isinstance(v, Tensor) and v.requires_grad for v in (x, delta, a, b, c, d, z, delta_bias, state))
    return _Scan.apply(x, delta, a, b, c, d, z, delta_bias, state, first, lengths, softplus, save)


def norm(y, residual, *, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid", eps=1e-6):
    """residual_norm, differentiable in every tensor."""
    return _Norm.apply(y, residual, gate, post_weight, scale, pre_weight, gate_act, eps)
