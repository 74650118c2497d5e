"""More operators of a policy with memory, as they are timed: a lighter recurrent cell, the matrix products around it and
the dropout on its residual stream, over the shapes in which an actor and a learner next to the simulator meet them.

  recurrence  gated linear recurrence, one state per channel: s = sigmoid(decay), a = exp(rate s),
              h = a h + sqrt(1 - a a) sigmoid(intake) x, y = h z sigmoid(z)
  projection  out = residual + act(x weight^T + bias), and its backward pass
  dropout     out = residual + x 2^16 / (2^16 - t) where the mask keeps x, t = round(p 2^16); the mask comes from Philox4x32-10,
              keyed by a seed and counted by (channel / 8, environment, step), so that a learner finds the actor's masks again

A case is a dict: `op` (which operator and form), `dtype` (f32 | bf16 | f16: activations; states and vectors of parameters are
f32), `steps`, `n` environments, `channels` (of a projection: inputs), and per operator `outputs`, `act`, `bias`, `save` (the
forward pass keeps what a backward pass needs), `weight` (rows: [outputs][inputs] | columns: a transposed [inputs][outputs]),
`residual` (none | same: of the activations' type | f32), `p`, `order` (time: [steps][n], as rollouts are | batch:
[n][steps], as recorded trajectories are), `ragged` (lengths from zero to `steps`), `starts` (episodes begin inside, mean length
180), `carried` (a state from before), `gate` (an output gate z).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPISODE_STEPS = 180.0       # mean length of an episode under random actions

RECURRENCE = {"order": "time", "ragged": False, "starts": False, "carried": False, "gate": False}
PROJECTION = {"order": "time", "act": "none", "bias": True, "residual": "none", "save": False, "weight": "rows"}
DROPOUT = {"order": "time", "residual": "none", "p": 0.1}


def _case(name, op, dtype, steps, n, channels, **how):
    base = RECURRENCE if op.startswith("recurrence") else PROJECTION if op.startswith("projection") else DROPOUT
    case = {"op": op, "dtype": dtype, "steps": steps, "n": n, "channels": channels, **base, **how}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one token of the smallest batch: an actor or an evaluation over 64 environments, where latency counts
        _case("recurrence_step_64", "recurrence_step", "f32", 1, 64, 512, starts=True, gate=True),
        # one token of the largest batch that the simulator is measured with
        _case("recurrence_step_65536", "recurrence_step", "bf16", 1, 65536, 512, starts=True, gate=True),
        # one whole episode of the longest length (10,000 steps) read again, one environment: all parallelism is along time
        _case("recurrence_prompt_10000", "recurrence_prompt", "f32", 10000, 1, 512),
        # a learner's update on a rollout of 4,096 environments: forward and backward
        _case("recurrence_train_4096", "recurrence_train", "bf16", 64, 4096, 512, starts=True, carried=True, gate=True),
        # an update on recorded trajectories of unequal lengths, batch first, odd sizes
        _case("recurrence_train_ragged", "recurrence_train", "f16", 1000, 37, 647, order="batch", ragged=True, carried=True, gate=True),
        # the embedding of the flat observation of Craftax-Classic (1,345 values) for 64 environments' actions
        _case("projection_64", "projection", "bf16", 1, 64, 1345, outputs=512, act="silu"),
        # the embedding of the full game's symbolic observation (8,268 values) in full precision, an odd number of rows
        _case("projection_8268", "projection", "f32", 3, 1001, 8268, outputs=256, act="relu"),
        # back from a block's inner width into a float32 residual stream, one token of 65,536 environments
        _case("projection_residual_65536", "projection", "f16", 1, 65536, 1024, outputs=512, residual="f32", weight="columns"),
        # a learner's update, into a block's inner width: forward, with what the backward pass needs
        _case("projection_262144", "projection", "bf16", 64, 4096, 512, outputs=1024, act="gelu_tanh", save=True),
        # and its backward pass
        _case("projection_back_262144", "projection_back", "bf16", 64, 4096, 512, outputs=1024, act="gelu_tanh"),
        # one token of 64 environments onto the residual stream
        _case("dropout_64", "dropout", "f32", 1, 64, 512, residual="same"),
        # a learner's update: forward and backward
        _case("dropout_train_4096", "dropout_train", "bf16", 64, 4096, 512, residual="same"),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["recurrence_step", "recurrence_prompt", "recurrence_train", "recurrence_train", "projection", "projection", "projection_back",
                     "dropout", "dropout_train"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    order = rng.choice(["time", "time", "batch"])
    if op.startswith("projection"):
        inputs = _log_int(rng, 16, 8268)
        outputs = rng.choice([18, 44, _log_int(rng, 16, 2048), _log_int(rng, 16, 2048)])       # heads: actions and a value
        if rng.random() < 0.5:
            inputs, outputs = (max(64, v // 64 * 64) for v in (inputs, outputs))
        act = rng.choice(["none", "relu", "silu", "gelu_tanh"])
        residual = rng.choice(["none", "none", "same", "f32"])
        # no more work than in the largest listed call (matrix units take float32 at a fraction of the others' rate)
        most = 262144 * 1024 * 512 // ((2 if op == "projection" else 1) * (12 if dtype == "f32" else 1)) // (inputs * outputs)
        rows = _log_int(rng, 1, max(1, min(262144, most, 262144 * 1536 // (inputs + 2 * outputs))))
        steps = _log_int(rng, 1, min(rows, 1000)) if rng.random() < 0.6 else 1
        how = {"outputs": outputs, "act": act, "bias": rng.random() < 0.8, "residual": residual, "order": order, "weight": rng.choice(["rows", "rows", "columns"])}
        if op == "projection":
            how["save"] = act != "none" and rng.random() < 0.5
        return _case(None, op, dtype, steps, max(1, rows // steps), inputs, **how)
    channels = _log_int(rng, 24, 2048)
    if rng.random() < 0.5:
        channels = max(64, channels // 64 * 64)
    if op.startswith("dropout"):
        steps = _log_int(rng, 1, 1000) if rng.random() < 0.7 else 1
        # no more values than in the largest update
        n = _log_int(rng, 1, max(1, min(65536, 60 * 4096 * 512 // (channels * steps * (2 if dtype == "f32" else 1)))))
        return _case(None, op, dtype, steps, n, channels, order=order, residual=rng.choice(["none", "same", "f32"]), p=rng.choice([0.02, 0.1, 0.25, 0.5]))
    how = {"starts": rng.random() < 0.5, "carried": rng.random() < 0.5, "gate": rng.random() < 0.5}
    if op == "recurrence_step":
        n = _log_int(rng, 1, max(1, min(65536, 65536 * 500 // channels)))
        return _case(None, op, dtype, 1, n, channels, **{**how, "starts": True})
    # sequences: no more steps and environments together than in the largest update
    steps = _log_int(rng, 1, 2000 if op == "recurrence_train" else 10000)
    n = _log_int(rng, 1, max(1, min(4096, 60 * 4096 * 512 // (channels * steps * (2 if dtype == "f32" else 1)))))
    return _case(None, op, dtype, steps, n, channels, **how, order=order, ragged=rng.random() < 0.4)


# ---- inputs ---------------------------------------------------------------------------------------

def _is_token(case):
    return case["op"].endswith("_step") or (case["steps"] == 1 and case["op"].split("_")[0] in ("projection", "dropout"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, D, T, n, op, token = DTYPES[case["dtype"]], case["channels"], case["steps"], case["n"], case["op"], _is_token(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda", dtype=torch.float32)

    def activation(width, spread=1.0, to=dtype, shift=0.0):
        if token:
            return (normal(n, width) * spread + shift).to(to)
        if case["order"] == "batch":
            return (normal(n, T, width) * spread + shift).to(to).transpose(0, 1)
        return (normal(T, n, width) * spread + shift).to(to)

    s = {"case": case, "op": op}
    kept = {"none": None, "same": dtype, "f32": torch.float32}[case.get("residual", "none")]
    if op.startswith("projection"):
        O = case["outputs"]
        s["x"] = activation(D)
        weight = (normal(O, D) / math.sqrt(D)).to(dtype)
        s["weight"] = weight if case["weight"] == "rows" else weight.t().contiguous().t()
        s["bias"] = 0.2 * normal(O) if case["bias"] else None
        if op == "projection":
            s["residual"] = None if kept is None else activation(O, 2.0, kept)
            return s
        s["pre"] = None
        if case["act"] != "none":                        # what the forward call keeps
            pre = s["x"].float() @ weight.float().t()
            s["pre"] = (pre if s["bias"] is None else pre + s["bias"]).to(dtype)
            if not token and case["order"] == "batch":
                s["pre"] = s["pre"].transpose(0, 1).contiguous().transpose(0, 1)
        s["dout"] = activation(O, 1.0, kept or dtype)
        return s
    if op.startswith("dropout"):
        values = random.Random(seed)
        s["mask_seed"], s["step"], s["env"] = values.getrandbits(64), values.randrange(1 << 40), values.randrange(1 << 20)
        s["x"] = activation(D)
        s["residual"] = None if kept is None else activation(D, 2.0, kept)
        s["dout"] = activation(D, 1.0, kept or dtype) if op == "dropout_train" else None
        return s

    s["first"] = s["lengths"] = None
    if case["starts"]:
        first = (uniform(T, n) < 1.0 / EPISODE_STEPS).to(torch.uint8)
        s["first"] = first[0] if token else first
    if case["ragged"]:
        lengths = (uniform(n) * (T + 1)).to(torch.int32).clamp_(max=T)
        if n > 2:
            lengths[1], lengths[n - 1] = 0, T
        s["lengths"] = lengths
    s["x"], s["decay"], s["intake"] = activation(D), activation(D, 1.0, dtype, 0.5), activation(D)
    s["z"] = activation(D) if case["gate"] else None
    s["rate"] = 8.0 * torch.log(0.9 + 0.099 * uniform(D))              # a step with its gate open keeps 0.43 to 0.99 of the state
    s["state"] = normal(n, D) if case["carried"] or token else None
    if op == "recurrence_train":
        s["dy"] = activation(D)
        s["dstate"] = normal(n, D) if case["carried"] else None
    if token:
        s["out_state"] = torch.empty_like(s["state"])
    return s


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2402_16801_amd import memory

    op, case = s["op"], s["case"]
    if op == "projection":
        out, pre = memory.projection(s["x"], s["weight"], s["bias"], residual=s["residual"], act=case["act"], save=case["save"])
        return (out, pre) if case["save"] else out
    if op == "projection_back":
        g = memory.projection_backward(s["dout"], s["x"], s["weight"], s["bias"], pre=s["pre"], act=case["act"])
        return tuple(v for v in (g.x, g.weight, g.bias) if v is not None)
    if op.startswith("dropout"):
        where = {"step": s["step"], "env": s["env"]}
        out = memory.residual_dropout(s["x"], case["p"], s["mask_seed"], residual=s["residual"], **where)
        if op == "dropout":
            return out
        return out, memory.residual_dropout_backward(s["dout"], case["p"], s["mask_seed"], dtype=s["x"].dtype, **where)
    if op == "recurrence_step":
        return memory.gated_recurrence_step(s["x"], s["decay"], s["intake"], s["rate"], s["state"], z=s["z"], first=s["first"], out_state=s["out_state"])
    how = {"z": s["z"], "state": s["state"], "first": s["first"], "lengths": s["lengths"]}
    y, h, saved = memory.gated_recurrence(s["x"], s["decay"], s["intake"], s["rate"], save=op == "recurrence_train", **how)
    if op == "recurrence_prompt":
        return y, h
    g = memory.gated_recurrence_backward(s["dy"], saved, s["x"], s["decay"], s["intake"], s["rate"], dstate=s["dstate"], **how)
    return tuple(v for v in (y, h, g.x, g.decay, g.intake, g.rate, g.z, g.state) if v is not None)


def _run_plain(s):
    op = s["op"]
    if op == "projection":
        return _plain_projection(s)
    if op == "projection_back":
        return _plain_projection_back(s)
    if op.startswith("dropout"):
        return _plain_dropout(s)
    if op == "recurrence_step":
        view = {k: v[None] if k in ("x", "decay", "intake", "z", "first") and v is not None else v for k, v in s.items()}
        y, h = _plain_recurrence(view)
        return y[0], h
    return _plain_recurrence(s)


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _act(p, act):
    if act == "relu":
        return torch.clamp(p, min=0.0)
    if act == "silu":
        return p * _sigmoid(p)
    if act == "gelu_tanh":
        return p * _sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (p + 0.044715 * p * p * p))
    return p


def _act_slope(p, act):
    if act == "relu":
        return (p > 0.0).float()
    if act == "silu":
        g = _sigmoid(p)
        return g * (1.0 + p * (1.0 - g))
    k = 2.0 * math.sqrt(2.0 / math.pi)
    g = _sigmoid(k * (p + 0.044715 * p * p * p))
    return g + p * g * (1.0 - g) * k * (1.0 + 3.0 * 0.044715 * p * p)


def _plain_projection(s):
    act, x = s["case"]["act"], s["x"]
    p = x.float() @ s["weight"].float().t()
    if s["bias"] is not None:
        p = p + s["bias"]
    out = _act(p, act)
    if s["residual"] is not None:
        out = s["residual"].float() + out
    out = out.to(x.dtype if s["residual"] is None else s["residual"].dtype)
    return (out, p.to(x.dtype)) if s["case"]["save"] else out


def _plain_projection_back(s):
    x, weight, like = s["x"].float(), s["weight"].float(), s["x"].dtype
    dp = s["dout"].float()
    if s["pre"] is not None:
        dp = dp * _act_slope(s["pre"].float(), s["case"]["act"])
    flat = dp.reshape(-1, dp.shape[-1])
    dx, dweight = dp @ weight, flat.t() @ x.reshape(-1, x.shape[-1])
    grads = (dx.to(like), dweight.to(like))
    return grads if s["bias"] is None else grads + (flat.sum(0),)


def _plain_keep(s):
    """Truth values [steps][n][channels]: eight halves of a counter's four words, the lower half first."""
    D = s["x"].shape[-1]
    token = s["x"].dim() == 2
    T, n = (1, s["x"].shape[0]) if token else s["x"].shape[:2]
    low, whole = 0xFFFFFFFF, torch.int64
    block = torch.arange((D + 7) // 8, device="cuda", dtype=whole)
    env = torch.arange(n, device="cuda", dtype=whole) + s["env"]
    step = torch.arange(T, device="cuda", dtype=whole) + s["step"]
    shape = (T, n, block.numel())
    c = [block.expand(shape), env[:, None].expand(shape), (step & low)[:, None, None].expand(shape), ((step >> 32) & low)[:, None, None].expand(shape)]
    k0, k1 = s["mask_seed"] & low, s["mask_seed"] >> 32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57                  # the lower 64 bits, signs and all
        c = [((p1 >> 32) & low) ^ c[1] ^ k0, p1 & low, ((p0 >> 32) & low) ^ c[3] ^ k1, p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    limit = int(math.floor(s["case"]["p"] * 65536.0 + 0.5))
    halves = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], -1)
    keep = (halves >= limit).reshape(T, n, -1)[..., :D]
    return (keep[0] if token else keep), 65536.0 / (65536 - limit)


def _plain_dropout(s):
    x = s["x"]
    keep, scale = _plain_keep(s)
    out = torch.where(keep, x.float() * scale, 0.0)
    if s["residual"] is not None:
        out = s["residual"].float() + out
    out = out.to(x.dtype if s["residual"] is None else s["residual"].dtype)
    if s["op"] == "dropout":
        return out
    return out, torch.where(keep, s["dout"].float() * scale, 0.0).to(x.dtype)


def _alive(s):
    """[steps][n][1] truth values: the steps before the end of each sequence; None where all are."""
    if s["lengths"] is None:
        return None
    t = torch.arange(s["x"].shape[0], device="cuda")
    return (t[:, None] < s["lengths"][None, :])[:, :, None]


def _running(a, b):
    """h_t = a_t h_(t-1) + b_t from h = 0, by doubling: after k turns a step holds what the last 2^k steps did."""
    a, b = a.clone(), b.clone()
    reach = 1
    while reach < a.shape[0]:
        b[reach:] += a[reach:] * b[:-reach]             # the right side is computed before it is added
        a[reach:] = a[reach:] * a[:-reach]
        reach *= 2
    return b


def _plain_recurrence(s):
    x, z, rate = s["x"].float(), s["z"], s["rate"]
    T, n, D = x.shape
    alive, train = _alive(s), s["op"] == "recurrence_train"
    g, q = _sigmoid(s["decay"].float()), _sigmoid(s["intake"].float())
    log_a = rate * g
    a, room = torch.exp(log_a), torch.sqrt(-torch.expm1(2.0 * log_a))
    new = room * q * x
    carry = a if s["first"] is None else torch.where((s["first"] != 0)[:, :, None], 0.0, a)
    if alive is not None:
        carry, new = torch.where(alive, carry, 1.0), torch.where(alive, new, 0.0)
    head = torch.zeros((n, D), device="cuda") if s["state"] is None else s["state"]
    taken = new.clone()
    taken[0] += carry[0] * head
    h = _running(carry, taken)
    gate = None if z is None else z.float()
    y = h if gate is None else h * gate * _sigmoid(gate)
    if alive is not None:
        y = torch.where(alive, y, 0.0)
    last = h[-1].clone()
    if not train:
        return y.to(s["x"].dtype), last

    like = s["x"].dtype
    dy = s["dy"].float()
    if alive is not None:
        dy = torch.where(alive, dy, 0.0)
    dz = None
    if gate is not None:
        sg = _sigmoid(gate)
        dz = dy * h * sg * (1.0 + gate * (1.0 - sg))
        dy = dy * gate * sg
    # G_t = dy_t + carry_(t+1) G_(t+1), from the end
    behind = torch.cat([carry[1:], torch.ones_like(carry[:1])]).flip(0)
    dh = dy.flip(0)
    if s["dstate"] is not None:
        dh[0] += s["dstate"]
    G = _running(behind, dh).flip(0)
    dhead = carry[0] * G[0]
    before = torch.cat([head[None], h[:-1]])
    if alive is not None:
        G = torch.where(alive, G, 0.0)
    dlog = G * (carry * before - q * x * a * a / room)
    through = G * room * q
    grads = [through.to(like), (dlog * rate * g * (1.0 - g)).to(like), (through * x * (1.0 - q)).to(like), (dlog * g).sum((0, 1))]
    if dz is not None:
        grads.append(dz.to(like))
    if s["state"] is not None:
        grads.append(dhead)
    return (y.to(like), last, *grads)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    T, n, D, op = (case[k] for k in ("steps", "n", "channels", "op"))
    rows = T * n
    kept = {"none": 0, "same": e, "f32": 4}[case.get("residual", "none")]
    if op.startswith("projection"):
        O = case["outputs"]
        slope = int(case["act"] != "none")
        if op == "projection":
            size = rows * D * e + O * D * e + rows * O * (kept + (kept or e) + (e if case["save"] else 0)) + 4 * O
            return {"bytes": size, "flops": rows * O * (2 * D + 2 + 8 * slope)}
        return {"bytes": rows * O * ((kept or e) + slope * e) + 2 * rows * D * e + 2 * O * D * e + 4 * O, "flops": rows * O * (4 * D + 1 + 12 * slope)}
    if op.startswith("dropout"):
        size = rows * D * (e + kept + (kept or e))
        if op == "dropout_train":
            size += rows * D * ((kept or e) + e)
        return {"bytes": size, "flops": rows * D * (3 if op == "dropout" else 5)}
    gate, carried = int(case["gate"]), int(case["carried"] or op == "recurrence_step")
    size = (4 + gate) * rows * D * e + (1 + carried) * n * D * 4 + D * 4
    flops = (20 + 5 * gate) * rows * D
    if op == "recurrence_train":
        size += (4 + gate) * rows * D * e + 2 * carried * n * D * 4 + D * 4
        flops += (40 + 10 * gate) * rows * D
    return {"bytes": size, "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    """Every output from its definition in 64 bits; gradients by automatic differentiation of the definition."""
    s = prepare(case, seed)
    if case["op"].startswith("projection"):
        return _exact_projection(case, s)
    if case["op"].startswith("dropout"):
        return _exact_dropout(case, s)
    return _exact_recurrence(case, s)


def _activation(case, p):
    f = torch.nn.functional
    return {"none": lambda v: v, "relu": f.relu, "silu": f.silu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[case["act"]](p)


def _exact_projection(case, s):
    x, weight = s["x"].double(), s["weight"].double()
    if case["op"] == "projection":
        p = torch.nn.functional.linear(x, weight, None if s["bias"] is None else s["bias"].double())
        out = _activation(case, p)
        if s["residual"] is not None:
            out = out + s["residual"].double()
        return (out, p) if case["save"] else out
    dp = s["dout"].double()
    if s["pre"] is not None:
        pre = s["pre"].double().requires_grad_(True)
        (dp,) = torch.autograd.grad(_activation(case, pre), pre, dp)
    rows = dp.reshape(-1, dp.shape[-1])
    out = (torch.matmul(dp, weight), torch.matmul(rows.transpose(0, 1), x.reshape(-1, x.shape[-1])))
    return out if s["bias"] is None else out + (rows.sum(0),)


def _exact_keep(case, s):
    """The mask, from 32-bit words taken apart into halves of 16 bits."""
    D = case["channels"]
    blocks = (D + 7) // 8
    T, n = case["steps"], case["n"]
    at = torch.arange(T * n * blocks, device="cuda")
    step = at // (n * blocks) + s["step"]
    words = [at % blocks, at // blocks % n + s["env"], step % 2 ** 32, step // 2 ** 32]
    key = [s["mask_seed"] % 2 ** 32, s["mask_seed"] // 2 ** 32]

    def product(word, factor):
        """(upper, lower) 32 bits of a 64-bit product"""
        low, high = word % 65536, word // 65536
        a, b = low * factor, high * factor                        # below 2^48 each
        middle = a // 65536 + b
        return middle // 65536, middle % 65536 * 65536 + a % 65536

    for turn in range(10):
        (h0, l0), (h1, l1) = product(words[0], 0xD2511F53), product(words[2], 0xCD9E8D57)
        k0, k1 = (key[0] + turn * 0x9E3779B9) % 2 ** 32, (key[1] + turn * 0xBB67AE85) % 2 ** 32
        words = [torch.bitwise_xor(torch.bitwise_xor(h1, words[1]), k0), l1, torch.bitwise_xor(torch.bitwise_xor(h0, words[3]), k1), l0]
    dropped = round(case["p"] * 65536)
    keep = torch.empty((T * n * blocks, 8), dtype=torch.bool, device="cuda")
    for j, w in enumerate(words):
        keep[:, 2 * j], keep[:, 2 * j + 1] = w % 65536 >= dropped, w // 65536 >= dropped
    return keep.view(T, n, blocks * 8)[:, :, :D].reshape(s["x"].shape), 65536 / (65536 - dropped)


def _exact_dropout(case, s):
    keep, scale = _exact_keep(case, s)
    factor = keep.double() * scale
    out = s["x"].double() * factor
    if s["residual"] is not None:
        out = out + s["residual"].double()
    return out if case["op"] == "dropout" else (out, s["dout"].double() * factor)


def _exact_recurrence(case, s):
    token, train = case["op"] == "recurrence_step", case["op"] == "recurrence_train"
    names = [k for k in ("x", "decay", "intake", "z") if s[k] is not None]
    leaf = {k: (s[k][None] if token else s[k]).double().requires_grad_(train) for k in names}
    rate = s["rate"].double().requires_grad_(train)
    T, n, D = leaf["x"].shape
    state = torch.zeros(n, D, device="cuda", dtype=torch.float64) if s["state"] is None else s["state"].double()
    state.requires_grad_(train)
    h, out = state, []
    for t in range(T):
        old = h
        if s["first"] is not None:
            old = old.masked_fill(((s["first"] if token else s["first"][t]) != 0)[:, None], 0.0)
        log_a = rate * torch.sigmoid(leaf["decay"][t])
        new = torch.exp(log_a) * old + torch.sqrt(-torch.expm1(2 * log_a)) * torch.sigmoid(leaf["intake"][t]) * leaf["x"][t]
        y = new if "z" not in leaf else new * torch.nn.functional.silu(leaf["z"][t])
        if s["lengths"] is not None:                              # steps behind the end leave the state as it is
            on = (t < s["lengths"])[:, None]
            new, y = torch.where(on, new, h), torch.where(on, y, torch.zeros_like(y))
        h = new
        out.append(y)
    y = torch.stack(out)
    if not train:
        return (y[0] if token else y), h
    outs, seeds = [y], [s["dy"].double()]
    if s["dstate"] is not None:
        outs.append(h)
        seeds.append(s["dstate"].double())
    wanted = [leaf["x"], leaf["decay"], leaf["intake"], rate] + [leaf[k] for k in names[3:]] + ([] if s["state"] is None else [state])
    return (y.detach(), h.detach(), *torch.autograd.grad(outs, wanted, seeds))
