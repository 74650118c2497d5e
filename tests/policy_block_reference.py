"""Plain 64-bit forms of the gated recurrence, the projection and the dropout from their definitions, on the CPU.  Gradients come from
automatic differentiation of these forms."""
import numpy as np
import torch


def recurrence(x, decay, intake, rate, z=None, state=None, first=None, lengths=None):
    T, n, D = x.shape
    h = torch.zeros(n, D, dtype=torch.float64) if state is None else state
    out = []
    for t in range(T):
        on = (torch.ones(n, dtype=torch.bool) if lengths is None else t < lengths)[:, None]

        def live(v):
            return torch.where(on, v[t], torch.zeros_like(v[t]))

        old = h if first is None else h.masked_fill((first[t] != 0)[:, None], 0.0)
        log_a = rate * torch.sigmoid(live(decay))
        new = torch.exp(log_a) * old + torch.sqrt(-torch.expm1(2 * log_a)) * torch.sigmoid(live(intake)) * live(x)
        y = new if z is None else new * live(z) * torch.sigmoid(live(z))
        h = torch.where(on, new, h)
        out.append(torch.where(on, y, torch.zeros_like(y)))
    return torch.stack(out), h


def act(v, name):
    if name == "relu":
        return torch.relu(v)
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    return v


def project(x, weight, bias=None, residual=None, act_name="none"):
    pre = x @ weight.t()
    if bias is not None:
        pre = pre + bias
    out = act(pre, act_name)
    return (out if residual is None else residual + out), pre


def keep_mask(seed, step, env, steps, n, channels, p):
    """bool [steps][n][channels] and the factor of what is kept: Philox4x32-10 in Python's whole numbers, eight channels at a time."""
    limit = int(p * 65536 + 0.5)
    keep = np.zeros((steps, n, (channels + 7) // 8 * 8), dtype=bool)
    for t in range(steps):
        for i in range(n):
            for block in range(keep.shape[2] // 8):
                c = [block, env + i, (step + t) & 0xFFFFFFFF, (step + t) >> 32]
                k = [seed & 0xFFFFFFFF, seed >> 32]
                for _ in range(10):
                    a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                    c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
                    k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
                for j in range(8):
                    keep[t, i, block * 8 + j] = (c[j // 2] >> (16 * (j % 2)) & 0xFFFF) >= limit
    return torch.from_numpy(keep[:, :, :channels].copy()), (65536 / (65536 - limit) if limit < 65536 else 0.0)


def dropout(x, keep, scale, residual=None):
    out = torch.where(keep, x * scale, torch.zeros_like(x))
    return out if residual is None else residual + out
