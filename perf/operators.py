"""The operators of a policy with memory, as they are timed: the parts of a recurrent policy block
that are no plain matrix product, over the shapes in which a learner next to the simulator meets them.

A policy acts one token per environment and step (`*_step`), reads prompts (an episode that is
evaluated, a recorded trajectory, ragged ones among them) and trains on rollouts laid out as the
simulator writes them, [steps][n], with the simulator's `done` flags as episode starts.

  conv   short causal convolution per channel, with a carried tail and silu
  scan   selective state space scan: h = exp(D A) h + D x B, y = (C . h + d x) silu(z)
  norm   norm after a block, gate, scale, residual, norm before the next block

A case is a dict: `op` (which operator and form), `dtype` (f32 | bf16 | f16: activations; parameters and
states are f32), `steps`, `n` environments (rows of a norm are steps * n), `channels`, and per operator
`states`, `groups` (channels of a group share B and C), `taps`, `order` (time: [steps][n], as rollouts
are | batch: [n][steps], as prompts are), `ragged` (lengths from zero to `steps`), `starts` (episodes
begin inside, mean length 180), `carried` (a state from before), `gate` (a gate tensor).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPISODE_STEPS = 180.0       # mean length of an episode under random actions
EPS = 1e-6

SEQUENCE = {"order": "time", "ragged": False, "starts": False, "carried": False, "gate": False}


def _case(name, op, dtype, steps, n, channels, states=16, groups=1, taps=4, **how):
    case = {"op": op, "dtype": dtype, "steps": steps, "n": n, "channels": channels, "states": states, "groups": groups, "taps": taps, **SEQUENCE, **how}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one token of the smallest batch: an actor or an evaluation over 64 environments, where latency counts
        _case("scan_step_64", "scan_step", "f32", 1, 64, 512, starts=True, gate=True),
        # one token of the largest batch that the simulator is measured with: 2 GiB of state read and written
        _case("scan_step_65536", "scan_step", "bf16", 1, 65536, 512, starts=True, gate=True),
        # one whole episode of the longest length (10,000 steps) read again, one environment: all parallelism is along time
        _case("scan_prompt_10000", "scan_prompt", "f32", 10000, 1, 512),
        # recorded trajectories of unequal lengths, batch first, two groups of channels, odd sizes
        _case("scan_prompt_ragged", "scan_prompt", "bf16", 1000, 37, 648, groups=2, order="batch", ragged=True, carried=True, gate=True),
        # a learner's update on a rollout of 4,096 environments: forward and backward
        _case("scan_train_4096", "scan_train", "bf16", 64, 4096, 512, starts=True, carried=True, gate=True),
        # a small learner in full precision with 32 states, odd sizes
        _case("scan_train_odd", "scan_train", "f32", 333, 19, 200, states=32, starts=True, carried=True),
        # one token of 4,096 environments through the convolution
        _case("conv_step_4096", "conv_step", "bf16", 1, 4096, 1024, starts=True),
        # ragged prompts, batch first, half precision
        _case("conv_prompt_ragged", "conv_prompt", "f16", 2000, 8, 1000, order="batch", ragged=True, carried=True),
        # the convolution of a learner's update, forward and backward
        _case("conv_train_4096", "conv_train", "bf16", 64, 4096, 512, starts=True, carried=True),
        # between two blocks of an actor's single token
        _case("norm_64", "norm", "bf16", 1, 64, 512, gate=True),
        # rows as wide as the flat observation of Craftax-Classic (1,345 values), full precision
        _case("norm_1345", "norm", "f32", 4, 5003, 1345),
        # between two blocks of a learner's update, forward and backward
        _case("norm_train_4096", "norm_train", "bf16", 64, 4096, 512, gate=True),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["scan_step", "scan_prompt", "scan_train", "scan_train", "conv_step", "conv_prompt", "conv_train", "norm", "norm_train"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    channels = _log_int(rng, 48, 1024)
    if rng.random() < 0.5:
        channels = max(64, channels // 64 * 64)
    groups = rng.choice([1, 1, 2, 4])
    channels = channels // groups * groups
    states = rng.choice([8, 16, 16, 32])
    taps = rng.choice([2, 3, 4, 4])
    how = {"starts": rng.random() < 0.5, "carried": rng.random() < 0.5, "gate": rng.random() < 0.5}
    if op.endswith("_step"):
        room = 65536 * 512 * 136 // (channels * (8 * states + 16))      # no more state than in the largest step
        return _case(None, op, dtype, 1, _log_int(rng, 1, max(1, min(65536, room))), channels, states, groups, taps, **{**how, "starts": True})
    # sequences: no more steps and environments together than in the largest update
    room = max(1, 60 * 4096 * 512 * 16 // (channels * (32 if op.startswith("scan") and states == 32 else 16)))
    steps = _log_int(rng, 1, 2000 if op == "scan_train" else 10000)
    n = _log_int(rng, 1, max(1, min(4096, room // steps)))
    if op.startswith("norm"):
        return _case(None, op, dtype, steps, n, channels, gate=how["gate"])
    how.update(order=rng.choice(["time", "batch"]), ragged=rng.random() < 0.4)
    return _case(None, op, dtype, steps, n, channels, states, groups, taps, **how)


# ---- inputs ---------------------------------------------------------------------------------------

def _sequence(case, gen, width, spread=1.0, groups=None):
    """Activations [steps][n][...], a view of [n][steps][...] where the order is batch first."""
    lead = (case["n"], case["steps"]) if case["order"] == "batch" else (case["steps"], case["n"])
    shape = lead + ((groups, width) if groups else (width,))
    v = (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * spread).to(DTYPES[case["dtype"]])
    return v.transpose(0, 1) if case["order"] == "batch" else v


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, D, N, G, K = DTYPES[case["dtype"]], case["channels"], case["states"], case["groups"], case["taps"]
    T, n, op = case["steps"], case["n"], case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda", dtype=torch.float32)

    s = {"case": case, "op": op}
    if op.startswith("norm"):
        s["y"], s["residual"] = _sequence(case, gen, D), _sequence(case, gen, D, 2.0)
        s["gate"] = _sequence(case, gen, D) if case["gate"] else None
        s["post_weight"], s["pre_weight"] = 1.0 + 0.1 * normal(D), 1.0 + 0.1 * normal(D)
        s["scale"] = 0.1 + 0.02 * normal(D)
        if op == "norm_train":
            s["dresidual"], s["du"] = _sequence(case, gen, D), _sequence(case, gen, D)
        return s

    step = op.endswith("_step")
    s["first"] = None
    if case["starts"]:
        first = (uniform(T, n) < 1.0 / EPISODE_STEPS).to(torch.uint8)
        s["first"] = first[0] if step else first
    s["lengths"] = None
    if case["ragged"]:
        lengths = (uniform(n) * (T + 1)).to(torch.int32).clamp_(max=T)
        if n > 2:
            lengths[1], lengths[n - 1] = 0, T
        s["lengths"] = lengths

    def activation(width, spread=1.0, groups=None):
        v = _sequence(case, gen, width, spread, groups)
        return v[0].contiguous() if step else v

    if op.startswith("conv"):
        s["x"] = activation(D)
        s["weight"], s["bias"] = normal(D, K) / math.sqrt(K), 0.1 * normal(D)
        s["state"] = normal(n, K - 1, D).to(dtype) if case["carried"] or step else None
        if op == "conv_train":
            s["dy"] = _sequence(case, gen, D)
            s["dstate"] = normal(n, K - 1, D).to(dtype) if case["carried"] else None
        if step:
            s["out_state"] = torch.empty_like(s["state"])
        return s

    s["x"], s["delta"] = activation(D), activation(D, 0.5)
    s["b"], s["c"] = activation(N, 1.0, G), activation(N, 1.0, G)
    s["z"] = activation(D) if case["gate"] else None
    s["a"] = -torch.arange(1, N + 1, device="cuda", dtype=torch.float32).repeat(D, 1) * (1.0 + 0.05 * normal(D, N))
    s["d"] = 1.0 + 0.1 * normal(D)
    size = torch.exp(uniform(D) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))       # steps of 0.001 to 0.1
    s["delta_bias"] = size + torch.log(-torch.expm1(-size))
    s["state"] = normal(n, D, N) if case["carried"] or step else None
    if op == "scan_train":
        s["dy"] = _sequence(case, gen, D)
        s["dstate"] = normal(n, D, N) if case["carried"] else None
    if step:
        s["out_state"] = torch.empty_like(s["state"])
    return s


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2402_16801_amd import memory

    op = s["op"]
    if op == "conv_step":
        return memory.causal_conv_step(s["x"], s["weight"], s["bias"], s["state"], first=s["first"], out_state=s["out_state"])
    if op in ("conv_prompt", "conv_train"):
        how = {"state": s["state"], "first": s["first"], "lengths": s["lengths"]}
        y, tail = memory.causal_conv(s["x"], s["weight"], s["bias"], **how)
        if op == "conv_prompt":
            return y, tail
        g = memory.causal_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], dstate=s["dstate"], **how)
        return (y, tail, g.x, g.weight, g.bias) + (() if s["state"] is None else (g.state,))
    if op == "scan_step":
        return memory.selective_scan_step(s["x"], s["delta"], s["a"], s["b"], s["c"], s["state"], d=s["d"], z=s["z"],
                                          delta_bias=s["delta_bias"], first=s["first"], out_state=s["out_state"])
    if op in ("scan_prompt", "scan_train"):
        how = {"d": s["d"], "z": s["z"], "delta_bias": s["delta_bias"], "state": s["state"], "first": s["first"], "lengths": s["lengths"]}
        y, h, saved = memory.selective_scan(s["x"], s["delta"], s["a"], s["b"], s["c"], save=op == "scan_train", **how)
        if op == "scan_prompt":
            return y, h
        g = memory.selective_scan_backward(s["dy"], saved, s["x"], s["delta"], s["a"], s["b"], s["c"], dstate=s["dstate"], **how)
        return tuple(v for v in (y, h, g.x, g.delta, g.a, g.b, g.c, g.d, g.z, g.delta_bias, g.state) if v is not None)
    how = {"gate": s["gate"], "post_weight": s["post_weight"], "scale": s["scale"], "pre_weight": s["pre_weight"], "eps": EPS}
    out = memory.residual_norm(s["y"], s["residual"], **how)
    if op == "norm":
        return out
    g = memory.residual_norm_backward(s["dresidual"], s["du"], s["y"], s["residual"], **how)
    return tuple(out) + tuple(v for v in (g.y, g.residual, g.gate, g.post_weight, g.scale, g.pre_weight) if v is not None)


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-torch.abs(v)))


def _alive(s):
    """[steps][n] truth values: the steps before the end of each sequence; None where all are."""
    if s["lengths"] is None:
        return None
    t = torch.arange(s["x"].shape[0], device="cuda")
    return t[:, None] < s["lengths"][None, :]


def _run_plain(s):
    op = s["op"]
    if op.startswith("norm"):
        return _plain_norm(s)
    if op.endswith("_step"):
        view = dict(s)
        for key in ("x", "delta", "b", "c", "z", "first"):
            if view.get(key) is not None:
                view[key] = view[key][None]
        y, state = (_plain_conv if op == "conv_step" else _plain_scan)(view)[:2]
        return y[0], state
    return _plain_conv(s) if op.startswith("conv") else _plain_scan(s)


def _plain_conv(s):
    """Shifted products. cat[j] is input j - (K - 1); episode numbers say which inputs a step still sees."""
    x, w, bias, K = s["x"], s["weight"], s["bias"], s["weight"].shape[1]
    T, n, D = x.shape
    head = torch.zeros((K - 1, n, D), device="cuda") if s["state"] is None else s["state"].float().transpose(0, 1)
    cat = torch.cat([head, x.float()])
    episode = torch.zeros((T, n), dtype=torch.int64, device="cuda") if s["first"] is None else torch.cumsum(s["first"].long(), 0)
    episode = torch.cat([torch.zeros((K - 1, n), dtype=torch.int64, device="cuda"), episode])
    alive = _alive(s)
    live = torch.ones((T, n), dtype=torch.bool, device="cuda") if alive is None else alive
    p = bias.expand(T, n, D)
    seen = []
    for k in range(K):
        seen.append((live & (episode[k:k + T] == episode[K - 1:]))[:, :, None])
        p = p + w[:, k] * torch.where(seen[k], cat[k:k + T], 0.0)
    gate = _sigmoid(p)
    y = torch.where(live[:, :, None], p * gate, 0.0).to(x.dtype)
    lengths = torch.full((n,), T, device="cuda", dtype=torch.int64) if s["lengths"] is None else s["lengths"].long()
    at = lengths[None, :] + torch.arange(K - 1, device="cuda")[:, None]                     # rows of cat that the tail holds
    last = torch.gather(episode, 0, lengths[None, :] + K - 2)
    kept = torch.gather(episode, 0, at) == last
    tail = torch.where(kept[:, :, None], torch.gather(cat, 0, at[:, :, None].expand(-1, -1, D)), 0.0).transpose(0, 1).to(x.dtype)
    if s["op"] != "conv_train":
        return y, tail

    dp = torch.where(live[:, :, None], s["dy"].float() * gate * (1.0 + p * (1.0 - gate)), 0.0)
    dcat = torch.zeros_like(cat)
    dw = torch.empty_like(w)
    for k in range(K):
        dcat[k:k + T] += torch.where(seen[k], w[:, k] * dp, 0.0)
        dw[:, k] = torch.where(seen[k], dp * cat[k:k + T], 0.0).sum((0, 1))
    if s["dstate"] is not None:
        add = torch.where(kept[:, :, None], s["dstate"].float().transpose(0, 1), 0.0)
        dcat.scatter_add_(0, at[:, :, None].expand(-1, -1, D), add)
    grads = (dcat[K - 1:].to(x.dtype), dw, dp.sum((0, 1)))
    return (y, tail) + grads + (() if s["state"] is None else (dcat[:K - 1].transpose(0, 1).to(x.dtype),))


def _plain_scan(s):
    """The recurrence step by step; for an update the states are kept and walked back."""
    x, a, (T, n, D) = s["x"].float(), s["a"], s["x"].shape
    G, N = s["b"].shape[2:]
    raw = s["delta"].float() + s["delta_bias"]
    delta = _softplus(raw)
    u = delta * x
    alive = _alive(s)
    train = s["op"] == "scan_train"

    def per_channel(v, t):
        return v[t].float()[:, :, None, :].expand(n, G, D // G, N).reshape(n, D, N)

    h = torch.zeros((n, D, N), device="cuda") if s["state"] is None else s["state"]
    before, after, sums = [], [], []
    for t in range(T):
        if s["first"] is not None:
            h = torch.where(s["first"][t][:, None, None] != 0, 0.0, h) if alive is None else \
                torch.where(((s["first"][t] != 0) & alive[t])[:, None, None], 0.0, h)
        if train:
            before.append(h)
        new = torch.exp(delta[t][:, :, None] * a) * h + u[t][:, :, None] * per_channel(s["b"], t)
        h = new if alive is None else torch.where(alive[t][:, None, None], new, h)
        if train:
            after.append(h)
        sums.append((h * per_channel(s["c"], t)).sum(-1))
    core = torch.stack(sums) + s["d"] * x
    gate = None if s["z"] is None else s["z"].float()
    y = core if gate is None else core * gate * _sigmoid(gate)
    if alive is not None:
        y = torch.where(alive[:, :, None], y, 0.0)
    y = y.to(s["x"].dtype)
    if not train:
        return y, h

    dy = s["dy"].float()
    dz = None
    if gate is not None:
        sg = _sigmoid(gate)
        dz = dy * core * sg * (1.0 + gate * (1.0 - sg))
        dy = dy * gate * sg
    if alive is not None:
        dy = torch.where(alive[:, :, None], dy, 0.0)
        dz = None if dz is None else torch.where(alive[:, :, None], dz, 0.0)
    g = torch.zeros((n, D, N), device="cuda") if s["dstate"] is None else s["dstate"]
    da = torch.zeros_like(a)
    du, ddelta, db, dc = torch.empty_like(x), torch.empty_like(x), [None] * T, [None] * T
    for t in reversed(range(T)):
        decay = torch.exp(delta[t][:, :, None] * a)
        g_t = g + per_channel(s["c"], t) * dy[t][:, :, None]
        if alive is not None:
            live = alive[t][:, None, None]
            keep, g_t = g, torch.where(live, g_t, 0.0)
        dc[t] = (after[t] * dy[t][:, :, None]).reshape(n, G, D // G, N).sum(2)
        db[t] = (g_t * u[t][:, :, None]).reshape(n, G, D // G, N).sum(2)
        du[t] = (g_t * per_channel(s["b"], t)).sum(-1)
        through = g_t * decay * before[t]
        ddelta[t] = (through * a).sum(-1)
        da += (through * delta[t][:, :, None]).sum(0)
        g = decay * g_t
        if s["first"] is not None:
            g = torch.where(s["first"][t][:, None, None] != 0, 0.0, g)
        if alive is not None:
            g = torch.where(live, g, keep)
    dx = delta * du + s["d"] * dy
    dpre = (ddelta + du * x) * _sigmoid(raw)
    like = s["x"].dtype
    out = [y, h, dx.to(like), dpre.to(like), da, torch.stack(db).to(like), torch.stack(dc).to(like), (dy * x).sum((0, 1))]
    if dz is not None:
        out.append(dz.to(like))
    out.append(dpre.sum((0, 1)))
    if s["state"] is not None:
        out.append(g)
    return tuple(out)


def _plain_norm(s):
    y, r = s["y"].float(), s["residual"].float()
    w1, w2, scale = s["post_weight"], s["pre_weight"], s["scale"]
    ry = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
    v = y * ry * w1
    act = _sigmoid(s["gate"].float()) if s["gate"] is not None else None
    o = v * scale if act is None else v * scale * act
    out = r + o
    ro = torch.rsqrt((out * out).mean(-1, keepdim=True) + EPS)
    u = out * ro * w2
    like = s["y"].dtype
    if s["op"] == "norm":
        return out.to(like), u.to(like)
    du = s["du"].float()
    t = du * w2
    unit = out * ro
    dr = s["dresidual"].float() + ro * (t - unit * (t * unit).mean(-1, keepdim=True))
    dv = dr * scale if act is None else dr * scale * act
    dscale = (dr * v if act is None else dr * v * act).sum((0, 1))
    yunit = y * ry
    q = dv * w1
    dy = ry * (q - yunit * (q * yunit).mean(-1, keepdim=True))
    grads = [dy.to(like), dr.to(like)]
    if act is not None:
        grads.append((dr * v * scale * act * (1.0 - act)).to(like))
    return (out.to(like), u.to(like), *grads, (dv * yunit).sum((0, 1)), dscale, (du * unit).sum((0, 1)))


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    T, n, D, N, G, K, op = (case[k] for k in ("steps", "n", "channels", "states", "groups", "taps", "op"))
    rows = T * n
    cells = rows * D
    if op.startswith("norm"):
        gate = int(case["gate"])
        read, write, flops = 2 + gate, 2, 10 + 4 * gate
        if op == "norm_train":
            read, write, flops = read + 2, write + 2 + gate, 3 * flops
        return {"bytes": (read + write) * cells * e + (6 if op == "norm_train" else 3) * D * 4, "flops": flops * cells}
    if op.startswith("conv"):
        tails = n * (K - 1) * D * e
        if op == "conv_train":
            carried = int(case["carried"])
            return {"bytes": 4 * cells * e + (1 + 3 * carried) * tails + 2 * D * (K + 1) * 4, "flops": (6 * K + 12) * cells}
        return {"bytes": 2 * cells * e + (1 + int(case["carried"] or op == "conv_step")) * tails + D * (K + 1) * 4, "flops": (2 * K + 4) * cells}
    gate, carried = int(case["gate"]), int(case["carried"] or op == "scan_step")
    shared, state, weights = 2 * rows * G * N * e, n * D * N * 4, D * (N + 2) * 4
    size = (3 + gate) * cells * e + shared + (1 + carried) * state + weights
    flops = (7 * N + 12) * cells
    if op == "scan_train":
        size += (3 + gate) * cells * e + shared + 2 * carried * state + weights
        flops += (20 * N + 20) * cells
    return {"bytes": size, "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    """Every output from its definition in 64 bits; gradients by automatic differentiation of the definition."""
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"].startswith("norm") else _exact_sequences(s)


def _doubles(s, keys):
    return {k: s[k].double().requires_grad_(True) for k in keys if s.get(k) is not None}


def _exact_norm(s):
    train = s["op"] == "norm_train"
    shape, D = s["y"].shape, s["y"].shape[-1]
    par = _doubles(s, ("post_weight", "scale", "pre_weight"))
    sums = {k: torch.zeros_like(v) for k, v in par.items()}
    rows = {k: s[k].reshape(-1, D) for k in ("y", "residual", "gate", "dresidual", "du") if s.get(k) is not None}
    parts = []
    count = max(1, (1 << 25) // D)
    for at in range(0, rows["y"].shape[0], count):
        v = _doubles({k: r[at:at + count] for k, r in rows.items()}, ("y", "residual", "gate"))
        branch = torch.nn.functional.rms_norm(v["y"], (D,), par["post_weight"], EPS) * par["scale"]
        if "gate" in v:
            branch = branch * torch.sigmoid(v["gate"])
        out = v["residual"] + branch
        u = torch.nn.functional.rms_norm(out, (D,), par["pre_weight"], EPS)
        got = [out.detach(), u.detach()]
        if train:
            wanted = list(v.values()) + list(par.values())
            seeds = [rows["dresidual"][at:at + count].double(), rows["du"][at:at + count].double()]
            grads = torch.autograd.grad([out, u], wanted, seeds)
            got += grads[:len(v)]
            for k, g in zip(par, grads[len(v):]):
                sums[k] += g
        parts.append(got)
    whole = [torch.cat(p).reshape(shape) for p in zip(*parts)]
    return tuple(whole) + (tuple(sums.values()) if train else ())


def _exact_sequences(s):
    """Some environments at a time, so that the kept states of an update fit."""
    op, scan = s["op"], s["op"].startswith("scan")
    step, train = op.endswith("_step"), op.endswith("_train")
    n = s["x"].shape[0 if step else 1]
    T, D = 1 if step else s["x"].shape[0], s["x"].shape[-1]
    sequences = [k for k in (("x", "delta", "b", "c", "z") if scan else ("x",)) if s[k] is not None]
    names = ("a", "d", "delta_bias") if scan else ("weight", "bias")
    par = _doubles(s, names)
    sums = {k: torch.zeros_like(v) for k, v in par.items()}
    N = s["a"].shape[1] if scan else 8
    count = max(1, (1 << 27 if train else 1 << 28) // (D * N * (T if train else 1)))
    parts = []
    for at in range(0, n, count):
        some = slice(at, min(n, at + count))
        leaf = _doubles({k: (s[k][some][None] if step else s[k][:, some]) for k in sequences}, sequences)
        if s["state"] is not None:
            leaf["state"] = s["state"][some].double().requires_grad_(True)
        first = None if s["first"] is None else (s["first"][some][None] if step else s["first"][:, some])
        lengths = None if s["lengths"] is None else s["lengths"][some]
        with torch.set_grad_enabled(train):
            y, last = (_define_scan if scan else _define_conv)(leaf, par, first, lengths)
        got = {"y": y.detach(), "last": last.detach()}
        if train:
            seeds = [s["dy"][:, some].double()]
            outs = [y]
            if s["dstate"] is not None:
                outs.append(last)
                seeds.append(s["dstate"][some].double())
            wanted = {**leaf, **par}
            grads = dict(zip(wanted, torch.autograd.grad(outs, list(wanted.values()), seeds, allow_unused=True)))
            for k in par:
                if grads[k] is not None:
                    sums[k] += grads[k]
            for k in leaf:
                got["d" + k] = torch.zeros_like(leaf[k]) if grads[k] is None else grads[k]
        parts.append(got)
    whole = {k: torch.cat([p[k] for p in parts], 0 if k in ("last", "dstate") else 1) for k in parts[0]}
    y = whole["y"][0] if step else whole["y"]
    if not train:
        return y, whole["last"]
    if scan:
        order = [whole["dx"], whole["ddelta"], sums["a"], whole["db"], whole["dc"], sums["d"], whole.get("dz"), sums["delta_bias"], whole.get("dstate")]
    else:
        order = [whole["dx"], sums["weight"], sums["bias"], whole.get("dstate")]
    return (y, whole["last"], *[v for v in order if v is not None])


def _define_conv(leaf, par, first, lengths):
    """A window of the last inputs that is pushed along, emptied where an episode begins."""
    x, K = leaf["x"], par["weight"].shape[1]
    T, n, D = x.shape
    window = leaf["state"] if "state" in leaf else x.new_zeros((n, K - 1, D))
    out = []
    for t in range(T):
        on = torch.ones(n, dtype=torch.bool, device="cuda") if lengths is None else t < lengths
        old = window
        if first is not None:
            old = torch.where((first[t] != 0)[:, None, None], torch.zeros_like(old), old)
        full = torch.cat([old, x[t][:, None]], 1)
        p = (full * par["weight"].t()).sum(1) + par["bias"]
        out.append(torch.where(on[:, None], torch.nn.functional.silu(p), torch.zeros_like(p)))
        window = torch.where(on[:, None, None], full[:, 1:], window)
    return torch.stack(out), window


def _define_scan(leaf, par, first, lengths):
    x, N = leaf["x"], par["a"].shape[1]
    T, n, D = x.shape
    each = D // leaf["b"].shape[2]
    h = leaf["state"] if "state" in leaf else x.new_zeros((n, D, N))
    out = []
    for t in range(T):
        size = torch.nn.functional.softplus(leaf["delta"][t] + par["delta_bias"], threshold=60.0)
        old = h
        if first is not None:
            old = old.masked_fill((first[t] != 0)[:, None, None], 0.0)
        b, c = (leaf[k][t].repeat_interleave(each, dim=1) for k in ("b", "c"))
        new = torch.exp(size[..., None] * par["a"]) * old + (size * x[t])[..., None] * b
        y = (new * c).sum(-1) + par["d"] * x[t]
        if "z" in leaf:
            y = y * torch.nn.functional.silu(leaf["z"][t])
        if lengths is None:
            h = new
        else:
            on = t < lengths
            h = torch.where(on[:, None, None], new, h)
            y = torch.where(on[:, None], y, torch.zeros_like(y))
        out.append(y)
    return torch.stack(out), h
