"""Plain 64-bit forms of the policy memory operators, step by step from their definitions, on the CPU.
Gradients come from automatic differentiation of these forms."""
import torch


def _on(lengths, t, n):
    return torch.ones(n, dtype=torch.bool) if lengths is None else t < lengths


def conv(x, weight, bias=None, state=None, first=None, lengths=None, silu=True):
    T, n, D = x.shape
    K = weight.shape[1]
    window = torch.zeros(n, K - 1, D, dtype=torch.float64) if state is None else state
    out = []
    for t in range(T):
        on = _on(lengths, t, n)
        old = window if first is None else window.masked_fill((first[t] != 0)[:, None, None], 0.0)
        x_t = torch.where(on[:, None], x[t], torch.zeros_like(x[t]))
        full = torch.cat([old, x_t[:, None]], 1)
        p = (full * weight.t()).sum(1)
        if bias is not None:
            p = p + bias
        if silu:
            p = p * torch.sigmoid(p)
        out.append(torch.where(on[:, None], p, torch.zeros_like(p)))
        window = torch.where(on[:, None, None], full[:, 1:], window)
    return torch.stack(out), window


def scan(x, delta, a, b, c, d=None, z=None, delta_bias=None, softplus=True, state=None, first=None, lengths=None):
    T, n, D = x.shape
    N, G = a.shape[1], b.shape[2]
    h = torch.zeros(n, D, N, dtype=torch.float64) if state is None else state
    out = []
    for t in range(T):
        on = _on(lengths, t, n)

        def live(v):
            keep = on.reshape(n, *[1] * (v.dim() - 1))
            return torch.where(keep, v, torch.zeros_like(v))

        pre = live(delta[t]) if delta_bias is None else live(delta[t]) + delta_bias
        size = torch.clamp(pre, min=0.0) + torch.log1p(torch.exp(-pre.abs())) if softplus else pre
        old = h if first is None else h.masked_fill((first[t] != 0)[:, None, None], 0.0)
        b_t, c_t = (live(v[t]).repeat_interleave(D // G, dim=1) for v in (b, c))
        new = torch.exp(size[..., None] * a) * old + (size * live(x[t]))[..., None] * b_t
        y = (new * c_t).sum(-1)
        if d is not None:
            y = y + d * live(x[t])
        if z is not None:
            y = y * live(z[t]) * torch.sigmoid(live(z[t]))
        h = torch.where(on[:, None, None], new, h)
        out.append(torch.where(on[:, None], y, torch.zeros_like(y)))
    return torch.stack(out), h


def norm(y, residual, gate=None, post_weight=None, scale=None, pre_weight=None, gate_act="sigmoid", eps=1e-6):
    branch = y
    if post_weight is not None:
        branch = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * post_weight
    if scale is not None:
        branch = branch * scale
    if gate is not None:
        branch = branch * {"sigmoid": torch.sigmoid, "silu": lambda g: g * torch.sigmoid(g), "linear": lambda g: g}[gate_act](gate)
    out = residual + branch
    u = out / torch.sqrt((out * out).mean(-1, keepdim=True) + eps)
    return out, u if pre_weight is None else u * pre_weight


def gradients(form, tensors, seeds, **how):
    """(outputs, {name: gradient}) of `form` for the given 64-bit tensors and the gradients `seeds` of its outputs (None: 0)."""
    leaf = {k: v.detach().clone().requires_grad_(True) for k, v in tensors.items() if v is not None}
    outs = form(**leaf, **how)
    used = [(o, s) for o, s in zip(outs, seeds) if s is not None]
    got = torch.autograd.grad([o for o, _ in used], list(leaf.values()), [s for _, s in used], allow_unused=True)
    return [o.detach() for o in outs], {k: torch.zeros_like(v) if g is None else g for (k, v), g in zip(leaf.items(), got)}
