"""The gated recurrence, the projection and the dropout against their definitions in 64 bits.

Tolerances of the recurrence as in test_gpu_memory.py: one rounding of the output's type, and 32 * 2^-24 * sqrt(m) of the tensor's largest
value for a sum of m terms in 32 bits, each right to some 16 roundings (the root of 1 - a * a, whose argument is right to 2^-21, is
one of them).  A projection adds m products, exact for 16-bit types, in 32 bits: the same with m = inputs.  Its backward pass rounds dp to
the type of the activations, which moves a sum by at most the type's rounding times the sum of the sizes of its terms.  Dropout
rounds a factor and one sum: 3 * 2^-24 of its terms.
"""
import math

import pytest
import torch

import policy_block_reference as ref
from memory_reference import gradients
from test_gpu_memory import ROUND, TYPES, Source, case_id, close, plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mem():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2402_16801_amd import memory
    return memory


# ---- gated recurrence ---------------------------------------------------------------------------------------

def rec_inputs(src, T, n, D, gate, carried, shift=0.0):
    t = {"x": src.seq(T, n, D), "decay": src.seq(T, n, D), "intake": src.seq(T, n, D), "z": src.seq(T, n, D) if gate else None,
         "rate": (-torch.exp(src.normal(D) - 2.0 + shift)).float().double(), "state": src.normal(n, D) if carried else None}
    return t


def rec_gpu(src, t):
    g = {k: src.gpu(t[k]) for k in ("x", "decay", "intake", "z")}
    g.update({k: plain(t[k]) for k in ("rate", "state")})
    return g


def rec_args(g):
    return [g[k] for k in ("x", "decay", "intake", "rate")], {k: g[k] for k in ("z", "state")}


REC_CASES = [
    # dtype, T, n, D, order, gate, carried, begins, ragged
    ("f32", 1, 1, 1, "time", False, False, 0.0, False),
    ("f32", 1, 5, 70, "time", True, True, 0.5, False),
    ("bf16", 1, 3, 64, "slice", True, True, 0.5, False),
    ("f16", 2, 3, 65, "batch", True, False, 0.3, False),
    ("f32", 7, 4, 3, "time", False, True, 0.3, True),
    ("bf16", 8, 4, 128, "time", True, True, 0.1, False),
    ("f32", 9, 3, 130, "slice", True, True, 0.2, True),
    ("f16", 33, 2, 66, "batch", True, True, 0.05, True),
    ("f32", 65, 2, 40, "batch", False, True, 0.05, True),
    ("bf16", 130, 3, 73, "slice", True, True, 0.03, True),
    ("f32", 300, 1, 64, "time", True, True, 0.0, False),
    ("f32", 301, 6, 70, "batch", True, False, 0.01, True),
    ("f16", 1025, 2, 33, "slice", False, True, 0.004, False),
    ("f32", 2050, 1, 130, "time", True, True, 0.001, True),
    ("bf16", 4099, 1, 64, "time", True, True, 0.0, False),
    ("f32", 3001, 2, 20, "batch", False, True, 0.0005, True),
]


def check_recurrence(mem, src, t, T, n, D, begins, ragged):
    first = src.flags(T, n, begins) if begins else None
    lengths = torch.tensor([(0, T, 1, T // 2)[(i + (n == 1)) % 4] for i in range(n)], dtype=torch.int32) if ragged else None
    dy, dstate = src.seq(T, n, D), src.normal(n, D) if t["state"] is not None else None
    (y, h), want = gradients(ref.recurrence, t, (dy, dstate), first=first, lengths=lengths)
    args, how = rec_args(rec_gpu(src, t))
    how["first"] = None if first is None else first.cuda()
    how["lengths"] = None if lengths is None else lengths.cuda()
    chain = min(T, 64)
    for save in (False, True):
        got_y, got_h, saved = mem.gated_recurrence(*args, save=save, **how)
        assert (saved is not None) == save
        close("y", got_y, y, chain)
        close("state", got_h, h, chain)
    got = mem.gated_recurrence_backward(src.gpu(dy), saved, *args, dstate=plain(dstate), **how)
    for name, value in got._asdict().items():
        if value is None:
            assert t[name] is None, name
            continue
        close("gradient of " + name, value, want[name], chain + (T * n if name == "rate" else 0))


@pytest.mark.parametrize("case", REC_CASES, ids=case_id)
def test_recurrence_and_its_gradients(mem, case):
    dtype, T, n, D, order, gate, carried, begins, ragged = case
    src = Source(T * 1000 + D, TYPES[dtype], order)
    check_recurrence(mem, src, rec_inputs(src, T, n, D, gate, carried), T, n, D, begins, ragged)


@pytest.mark.parametrize("dtype,T,n,D,ragged", [("f32", 13, 2500, 260, False), ("bf16", 20, 2100, 515, True), ("f16", 9, 70001, 6, False)])
def test_recurrence_of_many_environments(mem, dtype, T, n, D, ragged):
    """Whole sequences with several channels per thread; the last ones, the first ones and some between."""
    src = Source(n, TYPES[dtype])
    t = rec_inputs(src, T, n, D, True, True)
    first, dy, dstate = src.flags(T, n, 0.05), src.seq(T, n, D), src.normal(n, D)
    lengths = torch.tensor([(0, T, 1, T // 2)[i % 4] for i in range(n)], dtype=torch.int32) if ragged else None
    args, how = rec_args(rec_gpu(src, t))
    how.update(first=first.cuda(), lengths=None if lengths is None else lengths.cuda())
    y, h, saved = mem.gated_recurrence(*args, save=True, **how)
    got = mem.gated_recurrence_backward(src.gpu(dy), saved, *args, dstate=plain(dstate), **how)
    some = torch.cat([torch.arange(0, 5), torch.arange(n // 2, n // 2 + 5), torch.arange(n - 5, n)])
    part = {k: v if k == "rate" else v[some] if k == "state" else v[:, some] for k, v in t.items()}
    (want_y, want_h), want = gradients(ref.recurrence, part, (dy[:, some], dstate[some]), first=first[:, some],
                                       lengths=None if lengths is None else lengths[some])
    close("y", y[:, some.cuda()], want_y, T)
    close("state", h[some.cuda()], want_h, T)
    for name in ("x", "decay", "intake", "z"):
        close("gradient of " + name, getattr(got, name)[:, some.cuda()], want[name], T)
    close("gradient of state", got.state[some.cuda()], want["state"], T)
    # the gradient of the rates: the sum of what the environments give alone
    total = torch.zeros(D, dtype=torch.float64)
    for at in range(0, n, 700):
        piece = slice(at, min(n, at + 700))
        a, w = rec_args({k: v if k == "rate" or v is None else v[piece].contiguous() if k == "state" else v[:, piece].contiguous() for k, v in rec_gpu(src, t).items()})
        w.update(first=first[:, piece].contiguous().cuda(), lengths=None if lengths is None else lengths[piece].cuda())
        _, _, kept = mem.gated_recurrence(*a, save=True, **w)
        total += mem.gated_recurrence_backward(src.gpu(dy[:, piece].contiguous()), kept, *a, dstate=plain(dstate[piece]), **w).rate.double().cpu()
    close("gradient of rate", got.rate, total, T * n)


@pytest.mark.parametrize("dtype,n,D", [("bf16", 3001, 136), ("f32", 9001, 61), ("f16", 2003, 131), ("bf16", 70001, 5)])
def test_recurrence_step_of_many_environments(mem, dtype, n, D):
    src = Source(n, TYPES[dtype])
    t = rec_inputs(src, 1, n, D, True, True)
    first = src.flags(1, n, 0.3)
    y, h = ref.recurrence(first=first, **t)
    args, how = rec_args(rec_gpu(src, t))
    state = how["state"]
    got_y, got_h = mem.gated_recurrence_step(*[a if a.dim() == 1 else a[0] for a in args], state, z=how["z"][0], first=first[0].cuda())
    assert got_h is state
    close("y", got_y, y[0], 1)
    close("state", state, h, 1)


def test_recurrence_steps_equal_the_sequence(mem):
    """Token by token with the state in place, and the same in one call."""
    src = Source(21, torch.bfloat16)
    T, n, D = 50, 9, 132
    args, how = rec_args(rec_gpu(src, rec_inputs(src, T, n, D, True, True)))
    first = src.flags(T, n, 0.1).cuda()
    y, h, _ = mem.gated_recurrence(*args, first=first, **how)
    state = how["state"].clone()
    for t in range(T):
        got, _ = mem.gated_recurrence_step(args[0][t], args[1][t], args[2][t], args[3], state, z=how["z"][t], first=first[t])
        assert float((got.float() - y[t].float()).abs().max()) <= 2 * ROUND[torch.bfloat16] * float(y[t].float().abs().max()), t
    assert float((state - h).abs().max()) <= 64 * 2.0 ** -24 * float(h.abs().max())


@pytest.mark.parametrize("T", [40, 400])
def test_recurrence_forgets_infinities_and_ignores_dead_steps(mem, T):
    """NaN and infinities in the state of an episode that is over, in the steps before the begin of another one, and behind the end
    of a sequence leave no trace elsewhere."""
    src = Source(11, torch.float32)
    n, D = 4, 70
    t = rec_inputs(src, T, n, D, True, True)
    first = torch.zeros(T, n, dtype=torch.uint8)
    first[0, 0] = first[T // 2, 1] = first[0, 2] = first[1, 2] = first[T - 1, 3] = 1
    lengths = torch.tensor([T, T, T - 7, T], dtype=torch.int32)
    dy, dstate = src.seq(T, n, D), src.normal(n, D)
    dy[:, 2][T - 7:] = 0.0
    (y, h), want = gradients(ref.recurrence, t, (dy, dstate), first=first, lengths=lengths)
    bad = {k: v.clone() for k, v in t.items()}
    bad["state"][0], bad["state"][2] = float("inf"), float("nan")
    for k in ("x", "decay", "intake", "z"):
        bad[k][T - 7:, 2] = float("nan")
    for value in (float("nan"), float("inf")):
        bad["x"][T // 2 - 3, 1] = value
        args, how = rec_args(rec_gpu(src, bad))
        dy_bad = dy.clone()
        dy_bad[T - 7:, 2] = float("nan")
        how.update(first=first.cuda(), lengths=lengths.cuda())
        got_y, got_h, saved = mem.gated_recurrence(*args, save=True, **how)
        got = mem.gated_recurrence_backward(src.gpu(dy_bad), saved, *args, dstate=plain(dstate), **how)
        close("state", got_h, h, 64)
        for i, steps in ((0, slice(0, T)), (1, slice(T // 2, T)), (2, slice(0, T)), (3, slice(0, T))):
            close("y", got_y[steps, i], y[steps, i], 64)
            for name in ("x", "decay", "intake", "z"):
                close("gradient of " + name, getattr(got, name)[steps, i], want[name][steps, i], 64)
        assert bool((got_y[T - 7:, 2] == 0).all()) and all(bool((getattr(got, k)[T - 7:, 2] == 0).all()) for k in ("x", "decay", "intake", "z"))
        assert bool((got.state[0] == 0).all()) and bool((got.state[2] == 0).all())


def test_recurrence_with_rates_and_gates_at_their_ends(mem):
    """Rates of 0 (a sum of nothing: the state stays), of -2^-40 to -2^10, minus infinity, and gates that are shut or open to the last digit."""
    src = Source(13, torch.float32)
    T, n = 40, 3
    rates = [0.0, -(2.0 ** -40), -(2.0 ** -20), -(2.0 ** -8), -0.25, -0.26, -8.0, -(2.0 ** 10), -float("inf")]
    D = len(rates)
    t = rec_inputs(src, T, n, D, False, True)
    t["rate"] = torch.tensor(rates, dtype=torch.float64)
    t["decay"][5], t["decay"][6], t["decay"][7] = 30.0, -30.0, -100.0
    args, how = rec_args(rec_gpu(src, t))
    y, h, saved = mem.gated_recurrence(*args, save=True, **how)
    t["rate"][-1] = -1e30                                        # forgets as much
    t["rate"][0] = -(2.0 ** -120)                                # keeps as much, and has a derivative
    dy = src.seq(T, n, D)
    (want_y, want_h), want = gradients(ref.recurrence, t, (dy, None))
    for c in range(D):                                           # channel by channel: sizes of their own
        close("y", y[..., c], want_y[..., c], T)
        close("state", h[..., c], want_h[..., c], T)
    got = mem.gated_recurrence_backward(src.gpu(dy), saved, *args, **how)
    for c in range(1, D - 1):
        for name in ("x", "decay", "intake"):
            close(f"gradient of {name}", getattr(got, name)[..., c], want[name][..., c], T)
    for value in got:
        assert value is None or bool(torch.isfinite(value).all())
    assert bool((got.x[..., 0] == 0).all()) and bool((got.decay[..., 0] == 0).all())


def test_recurrence_gradients_against_differences(mem):
    """Along a random direction of all inputs: central differences of step 2^-7 of the kernel's own forward pass.  Their error: the third
    derivative, some units times 2^-14 / 6, and the roundings of some 5,000 outputs of size 1 over 2^-7; together below 1 percent of
    slopes that are of the order of sqrt(5,000).  Rates are kept away from 0, where the root has no derivative."""
    src = Source(31, torch.float32)
    T, n, D = 18, 4, 70
    t = rec_inputs(src, T, n, D, True, True, shift=1.0)
    first = src.flags(T, n, 0.05).cuda()
    w, wh = src.seq(T, n, D), src.normal(n, D)
    way = {k: 0.3 * src.normal(*v.shape) for k, v in t.items()}
    way["rate"] = way["rate"] * t["rate"]

    def loss(shift, save=False):
        args, how = rec_args({k: plain(v + shift * way[k]) for k, v in t.items()})
        y, h, saved = mem.gated_recurrence(*args, first=first, save=save, **how)
        value = float((y.double().cpu() * w).sum() + (h.double().cpu() * wh).sum())
        return (value, args, how, saved) if save else value

    _, args, how, saved = loss(0.0, save=True)
    got = mem.gated_recurrence_backward(plain(w), saved, *args, first=first, dstate=plain(wh), **how)._asdict()
    slope = sum(float((got[k].double().cpu() * way[k]).sum()) for k in way)
    step = 2.0 ** -7
    difference = (loss(step) - loss(-step)) / (2 * step)
    size = math.sqrt(sum(float((got[k].double().cpu() * way[k]).pow(2).sum()) for k in way))
    assert abs(slope - difference) <= 0.01 * size, (slope, difference, size)


def test_recurrence_beyond_two_to_the_31_elements(mem):
    """Offsets pass 32 bits; the last environments come out as they do alone."""
    T, n, D = 600, 3600, 1024
    src = Source(41, torch.bfloat16)
    t = rec_inputs(src, T, 2, D, False, False)
    g = rec_gpu(src, t)
    big = {}
    for k in ("x", "decay", "intake"):
        big[k] = torch.zeros(T, n, D, dtype=torch.bfloat16, device="cuda")
        big[k][:, -2:] = g[k]
    y, h, saved = mem.gated_recurrence(big["x"], big["decay"], big["intake"], g["rate"], save=True)
    small, small_h, kept = mem.gated_recurrence(g["x"], g["decay"], g["intake"], g["rate"], save=True)
    unit = 2 * ROUND[torch.bfloat16]
    assert float((y[:, -2:].float() - small.float()).abs().max()) <= unit * float(small.float().abs().max())
    assert bool((y[:, :-2] == 0).all())
    dy = torch.zeros_like(y)
    dy[:, -2:] = small
    got = mem.gated_recurrence_backward(dy, saved, big["x"], big["decay"], big["intake"], g["rate"])
    want = mem.gated_recurrence_backward(small, kept, g["x"], g["decay"], g["intake"], g["rate"])
    for name in ("x", "decay", "intake"):
        a, b = getattr(got, name)[:, -2:].float(), getattr(want, name).float()
        assert float((a - b).abs().max()) <= unit * float(b.abs().max()), name


# ---- projection ----------------------------------------------------------------------------------------------

PROJECT_CASES = [
    # dtype, T, n, inputs, outputs, act, residual, order, bias, weight by columns
    ("f32", 1, 1, 1, 1, "none", None, "time", False, False),
    ("bf16", 1, 1, 7, 3, "silu", "same", "time", True, True),
    ("f16", 1, 3, 1, 5, "relu", "f32", "time", True, False),
    ("f32", 1, 64, 1345, 18, "silu", "same", "time", True, False),
    ("bf16", 1, 64, 1345, 512, "gelu_tanh", "f32", "time", True, False),
    ("bf16", 2, 17, 63, 44, "silu", "same", "slice", True, True),
    ("f32", 3, 5, 65, 33, "gelu_tanh", None, "batch", False, True),
    ("f16", 1, 16, 64, 16, "none", "same", "time", True, False),
    ("bf16", 1, 257, 129, 260, "relu", "f32", "time", True, False),
    ("f32", 7, 150, 200, 270, "silu", "f32", "batch", True, False),
    ("bf16", 5, 333, 96, 640, "none", "f32", "slice", True, True),
    ("f16", 9, 301, 513, 300, "gelu_tanh", "same", "batch", True, False),
    ("bf16", 40, 257, 64, 128, "silu", None, "time", True, False),
    ("f32", 2, 2050, 72, 520, "none", None, "slice", True, True),
    ("bf16", 3, 4500, 256, 384, "gelu_tanh", "same", "time", True, False),
    ("f16", 1, 33000, 40, 136, "relu", "f32", "time", False, True),
    ("bf16", 1, 200, 8268, 256, "none", None, "time", True, False),
    ("f32", 1, 700, 4100, 70, "relu", None, "time", True, False),
]


def project_inputs(src, T, n, inputs, outputs, bias):
    return {"x": src.seq(T, n, inputs), "weight": src.normal(outputs, inputs, spread=inputs ** -0.5, dtype=src.dtype),
            "bias": src.normal(outputs) if bias else None}


def near(what, got, want, slack):
    """Off by no more than one rounding of the type and `slack`, a tensor."""
    got64 = got.detach().cpu().double()
    assert got64.shape == want.shape, (what, got64.shape, want.shape)
    over = (got64 - want).abs() - (ROUND[got.dtype] * (want.abs() + slack) + slack + 2.0 ** -25)
    assert bool((over <= 0).all()), f"{what}: off by {float((got64 - want).abs().max()):.3g}, worst {float(over.max()):.3g} over what is allowed"


def sums(terms, count):
    """What `count` additions in 32 bits may move a sum whose terms' sizes add up to `terms`: with terms of either sign the sums on the way are about
    terms / sqrt(count), and sqrt(count) of their roundings are left, one rounding of `terms`; four times that, and 16 more for few."""
    return terms * 2.0 ** -24 * (4 + 16 / math.sqrt(max(count, 1)))


@pytest.mark.parametrize("case", PROJECT_CASES, ids=case_id)
def test_projection_and_its_gradients(mem, case):
    dtype, T, n, I, O, act, residual, order, bias, columns = case
    src = Source(T * 1000 + I + O, TYPES[dtype], order)
    t = project_inputs(src, T, n, I, O, bias)
    wide = {None: None, "same": TYPES[dtype], "f32": torch.float32}[residual]
    res = None if wide is None else src.normal(T, n, O, dtype=wide)
    want, want_pre = ref.project(**t, residual=res, act_name=act)
    x, weight, b = src.gpu(t["x"]), t["weight"].to("cuda", TYPES[dtype]), plain(t["bias"])
    if columns:
        weight = weight.t().contiguous().t()
    out, pre = mem.projection(x, weight, b, residual=src.gpu(res, wide), act=act, save=True)
    assert out.dtype == (wide or TYPES[dtype]) and pre.dtype == TYPES[dtype]
    terms = t["x"].abs() @ t["weight"].abs().t() + (0 if t["bias"] is None else t["bias"].abs())
    off = sums(terms, I)
    near("pre", pre, want_pre, off)
    near("out", out, want, 1.2 * off + 2.0 ** -21 * (want.abs() + want_pre.abs()))          # the slope of an activation is below 1.2
    alone, nothing = mem.projection(x, weight, b, residual=src.gpu(res, wide), act=act)
    assert nothing is None and torch.equal(alone, out)

    unit = ROUND[TYPES[dtype]]
    dout = src.normal(T, n, O, dtype=wide or TYPES[dtype])
    given = pre.detach().cpu().double().requires_grad_(True)
    (dp,) = torch.autograd.grad(ref.act(given, act), given, dout)
    rows, flat = dp.reshape(-1, O), t["x"].reshape(-1, I)
    rounded = 1.1 * unit if act != "none" or wide not in (None, TYPES[dtype]) else 0.0          # dp as the products take it
    slope = 2.0 ** -21
    for float_weight in (False, True):
        g = mem.projection_backward(src.gpu(dout, wide or TYPES[dtype]), x, weight, b, pre=None if act == "none" else pre, act=act, float_weight=float_weight)
        size = dp.abs() @ t["weight"].abs()
        near("gradient of x", g.x, dp @ t["weight"], size * (rounded + slope) + sums(size, O))
        size = rows.abs().t() @ flat.abs()
        near("gradient of weight", g.weight, rows.t() @ flat, size * (rounded + slope) + sums(size, T * n))
        assert g.weight.dtype == (torch.float32 if float_weight else TYPES[dtype])
        assert (g.bias is None) == (b is None)
        if b is not None:
            size = rows.abs().sum(0)
            near("gradient of bias", g.bias, rows.sum(0), size * slope + sums(size, T * n))
    less = mem.projection_backward(src.gpu(dout, wide or TYPES[dtype]), x, weight, None, pre=pre, act=act, want_x=False)
    assert less.x is None and less.bias is None and torch.equal(less.weight.float(), mem.projection_backward(
        src.gpu(dout, wide or TYPES[dtype]), x, weight, b, pre=pre, act=act).weight.float())
    less = mem.projection_backward(src.gpu(dout, wide or TYPES[dtype]), x, weight, b, pre=pre, act=act, want_weight=False)
    assert less.weight is None and torch.equal(less.x, g.x)


def test_projection_of_exact_values(mem):
    """Small whole numbers: every product and sum is exact, so every value has to be, wherever it lies in a tile."""
    gen = torch.Generator().manual_seed(7)
    for dtype, rows, I, O in (("bf16", 1300, 100, 700), ("f16", 33333, 72, 130), ("f32", 1301, 37, 900), ("bf16", 17, 333, 50), ("bf16", 260, 4001, 130)):
        x = torch.randint(-2, 3, (rows, I), generator=gen).double()
        w = torch.randint(-2, 3, (O, I), generator=gen).double()
        d = torch.randint(-1, 2, (rows, O), generator=gen).double()
        gx, gw, gd = (v.to("cuda", TYPES[dtype]) for v in (x, w, d))
        zero = torch.zeros(rows, O, device="cuda")
        for weight in (gw, gw.t().contiguous().t()):
            out, _ = mem.projection(gx, weight, residual=zero)
            assert torch.equal(out.cpu().double(), x @ w.t()), (dtype, rows)
        g = mem.projection_backward(gd, gx, gw, torch.zeros(O, device="cuda"), float_weight=True)
        assert torch.equal(g.weight.cpu().double(), d.t() @ x), (dtype, rows)
        assert torch.equal(g.bias.cpu().double(), d.sum(0)), (dtype, rows)
        assert torch.equal(g.x.cpu().double(), (d @ w).to(TYPES[dtype]).double()), (dtype, rows)


def test_projection_of_exact_values_in_large_tiles(mem):
    """The same where operands go straight to LDS: more columns than biases are kept for, tiles that end inside the matrix, rows that are copied to where
    they can be read (odd counts, a slice of wider rows, environments first), sums in parts."""
    gen = torch.Generator(device="cuda").manual_seed(11)

    def whole(most, *shape):
        return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").double()

    for dtype, T, n, I, O, layout in (("bf16", 1, 1500, 64, 4200, "time"), ("f16", 1, 4000, 64, 4200, "time"), ("bf16", 1, 4000, 72, 4100, "time"),
                                      ("bf16", 60, 351, 701, 300, "time"), ("f16", 50, 410, 704, 300, "slice"), ("bf16", 300, 70, 704, 301, "batch"),
                                      ("bf16", 1, 900, 8192, 520, "time"), ("f16", 40, 400, 512, 264, "batch")):
        kind = TYPES[dtype]
        x, w, b, d, res = whole(2, T, n, I), whole(1, O, I), whole(30, O), whole(1, T, n, O), whole(30, T, n, O)
        if layout == "batch":
            gx, gres, gd = (v.to(kind).transpose(0, 1).contiguous().transpose(0, 1) for v in (x, res, d))
        elif layout == "slice":
            gx = torch.full((T, n + 3, I), float("nan"), dtype=kind, device="cuda")[:, 2:n + 2].copy_(x)
            gres, gd = res.to(kind), torch.full((T, n, O + 8), float("nan"), dtype=kind, device="cuda")[..., :O].copy_(d)
        else:
            gx, gres, gd = x.to(kind), res.to(kind), d.to(kind)
        out, pre = mem.projection(gx, w.to(kind), b.float(), residual=gres, act="relu", save=True)
        want = x.reshape(-1, I) @ w.t() + b
        assert torch.equal(pre.double(), want.to(kind).double().reshape(T, n, O)), (dtype, T, n, I, O)
        exact = (want.clamp(min=0.0).reshape(T, n, O) + res).to(kind).double()
        assert torch.equal(out.double(), exact), (dtype, T, n, I, O)
        for weight in (w.to(kind), w.to(kind).t().contiguous().t()):
            g = mem.projection_backward(gd, gx, weight, b.float(), float_weight=True)
            flat = d.reshape(-1, O)
            assert torch.equal(g.weight.double(), flat.t() @ x.reshape(-1, I)), (dtype, T, n, I, O)
            assert torch.equal(g.bias.double(), flat.sum(0)), (dtype, T, n, I, O)
            assert torch.equal(g.x.double(), (d @ w).to(kind).double()), (dtype, T, n, I, O)


@pytest.mark.parametrize("rows,I,O", [(700, 300, 400), (3000, 500, 24), (40, 2000, 1100)])
def test_projection_of_float32_at_the_ends_of_its_range(mem, rows, I, O):
    """Float32 values go through the matrix units in three parts: infinities, NaN and the largest numbers come out as from a plain sum, in their
    rows alone, and every other value of the same tile to the same digits as without them.  Very large and very small rows keep their digits."""
    src = Source(rows, torch.float32)
    x, w = src.normal(rows, I), src.normal(O, I, spread=I ** -0.5)
    x[1], x[2] = x[1] * 2.0 ** 100, x[2] * 2.0 ** -80
    want = x @ w.t()
    off = sums(x.abs() @ w.abs().t(), I)
    spoilt = x.clone()
    spoilt[5, I - 1], spoilt[9, 0], spoilt[11, I // 2] = float("inf"), float("nan"), -float("inf")
    spoilt[13] = 0.0
    spoilt[13, 3] = torch.finfo(torch.float32).max
    for given in (x, spoilt):
        out, _ = mem.projection(plain(given), plain(w))
        got = out.cpu().double()
        for m in range(rows):
            if given is x or m not in (5, 9, 11, 13):
                assert bool(((got[m] - want[m]).abs() <= 2 * ROUND[torch.float32] * want[m].abs() + 2 * off[m]).all()), m
    assert bool(got[9].isnan().all()) and torch.equal(got[5], float("inf") * w[:, I - 1].sign()) and torch.equal(got[11], -float("inf") * w[:, I // 2].sign())
    exact = torch.finfo(torch.float32).max * w[:, 3]
    assert bool(((got[13] - exact).abs() <= 2 * ROUND[torch.float32] * exact.abs()).all())
    d = src.normal(rows, O)
    g = mem.projection_backward(plain(d), plain(spoilt), plain(w))
    fine = [c for c in range(I) if c not in (0, 3, I // 2, I - 1)]
    keep = spoilt[:, fine]
    size = d.abs().t() @ keep.abs()
    assert bool(((g.weight.cpu().double()[:, fine] - d.t() @ keep).abs() <= 2 * sums(size, rows)).all())
    assert bool(g.weight[:, 0].isnan().all()) and bool(g.weight[:, I - 1].isinf().all())


@pytest.mark.parametrize("rows", [(7, 5), (60, 70), (90, 500)])
def test_projection_of_tensors_in_different_orders(mem, rows):
    """x lies environments first, residual and the gradient steps first, pre in a slice: whole numbers, so everything is exact."""
    T, n = rows
    gen = torch.Generator(device="cuda").manual_seed(T)
    I, O = 136, 264

    def whole(most, *shape):
        return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").double()

    for dtype in TYPES.values():
        x, w, d, res = whole(2, T, n, I), whole(1, O, I), whole(1, T, n, O), whole(9, T, n, O)
        gx = x.to(dtype).transpose(0, 1).contiguous().transpose(0, 1)
        out, pre = mem.projection(gx, w.to(dtype), residual=res.float(), act="relu", save=True)
        want = x @ w.t()
        assert torch.equal(out.double(), want.clamp(min=0.0) + res) and torch.equal(pre.double(), want)
        kept = torch.full((T, n + 1, O + 3), float("nan"), dtype=dtype, device="cuda")[:, 1:, 2:O + 2].copy_(pre)
        g = mem.projection_backward(d.float(), gx, w.to(dtype), torch.zeros(O, device="cuda"), pre=kept, act="relu", float_weight=True)
        dp = d * (want > 0)
        assert torch.equal(g.x.double(), (dp @ w).to(dtype).double())
        assert torch.equal(g.weight.double(), dp.reshape(-1, O).t() @ x.reshape(-1, I))
        assert torch.equal(g.bias.double(), dp.reshape(-1, O).sum(0))


def test_projection_leaves_what_is_beside_its_outputs(mem):
    """At the C entry: outputs inside wider rows, everything around them as it was; and inputs beside NaN."""
    from paper_2402_16801_amd import binding as cx
    lib = cx.load()
    for rows, I, O in ((3, 9, 5), (70, 100, 77), (1500, 65, 203), (5000, 33, 140)):
        x = torch.full((rows + 1, I + 5), float("nan"), dtype=torch.bfloat16, device="cuda")
        w = torch.full((O + 1, I + 3), float("nan"), dtype=torch.bfloat16, device="cuda")
        x[:rows, 2:2 + I], w[:O, 1:1 + I] = torch.randn(rows, I, device="cuda"), torch.randn(O, I, device="cuda")
        out = torch.full((rows + 2, O + 9), 7.0, dtype=torch.bfloat16, device="cuda")
        pre = torch.full((rows + 2, O + 9), 7.0, dtype=torch.bfloat16, device="cuda")
        a = cx.ProjectionArgs(dtype=1, out_dtype=1, act=2, steps=1, n=rows, inputs=I, outputs=O, weight=w[0, 1:].data_ptr(), weight_row=I + 3, weight_column=1,
                              x=x[0, 2:].data_ptr(), x_env=I + 5, out=out[1, 4:].data_ptr(), out_env=O + 9, pre=pre[1, 4:].data_ptr(), pre_env=O + 9)
        need = lib.craftax_projection_workspace_bytes(a, 0)
        work = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = work.data_ptr(), need
        assert lib.craftax_projection(a, torch.cuda.current_stream().cuda_stream) == 0
        want, want_pre = mem.projection(x[:rows, 2:2 + I], w[:O, 1:1 + I].contiguous(), act="silu", save=True)
        for got, exp in ((out, want), (pre, want_pre)):
            assert torch.equal(got[1:rows + 1, 4:4 + O], exp) and bool(torch.isfinite(exp).all())
            got[1:rows + 1, 4:4 + O] = 7.0
            assert bool((got == 7.0).all())


def test_projection_gradients_against_differences(mem):
    """As for the recurrence: a step of 2^-7 along a random direction, 1 percent."""
    src = Source(33, torch.float32)
    T, n, I, O = 3, 11, 70, 37
    t = project_inputs(src, T, n, I, O, True)
    t["residual"] = src.seq(T, n, O)
    w = src.seq(T, n, O)
    way = {k: 0.3 * src.normal(*v.shape, spread=I ** -0.5 if k == "weight" else 1.0) for k, v in t.items()}
    for act in ("silu", "gelu_tanh"):
        def at(shift):
            return {k: plain(v + shift * way[k]) for k, v in t.items()}

        def loss(shift):
            g = at(shift)
            return float((mem.project(g["x"], g["weight"], g["bias"], residual=g["residual"], act=act).double().cpu() * w).sum())

        leaf = {k: v.requires_grad_(True) for k, v in at(0.0).items()}
        got = torch.autograd.grad(mem.project(leaf["x"], leaf["weight"], leaf["bias"], residual=leaf["residual"], act=act), list(leaf.values()), plain(w))
        parts = [float((g.double().cpu() * way[k]).sum()) for k, g in zip(leaf, got)]
        size = math.sqrt(sum(float((g.double().cpu() * way[k]).pow(2).sum()) for k, g in zip(leaf, got)))
        step = 2.0 ** -7
        assert abs(sum(parts) - (loss(step) - loss(-step)) / (2 * step)) <= 0.01 * size


def test_projection_of_values_at_the_ends_of_their_range(mem):
    """Activations of large values are 0 or the value, their slopes 0 or 1; NaN stays NaN and in its row."""
    big = torch.tensor([-1e30, -300.0, -40.0, -0.0, 0.0, 40.0, 300.0, 1e30, float("nan")], device="cuda")
    for act in ("none", "relu", "silu", "gelu_tanh"):
        out, pre = mem.projection(big[:, None].contiguous(), torch.ones(1, 1, device="cuda"), act=act, save=True)
        out, pre = out[:, 0], pre[:, 0]
        assert torch.equal(pre[:8], big[:8]) and bool(pre[8].isnan()) and bool(out[8].isnan())
        if act != "none":
            assert bool((out[:2].abs() <= 1e-35).all()) and torch.equal(out[5:8], big[5:8])
        g = mem.projection_backward(torch.ones(9, 1, device="cuda"), big[:, None].contiguous(), torch.ones(1, 1, device="cuda"), pre=pre[:, None].contiguous(), act=act)
        slope = g.x[:, 0]
        assert bool(slope[8].isnan()) or act == "none"
        if act != "none":
            assert bool((slope[:2] == 0).all()) and bool((slope[5:8] == 1).all()), act
    rows = torch.randn(40, 70, device="cuda")
    rows[7, 3] = float("nan")
    out, _ = mem.projection(rows, torch.randn(50, 70, device="cuda"))
    assert bool(out[7].isnan().all()) and bool(torch.isfinite(torch.cat([out[:7], out[8:]])).all())


def test_projection_beyond_two_to_the_31_elements(mem):
    """Outputs and inputs whose offsets pass 32 bits; the last rows come out as they do alone, and gradients of the weight sum over all rows."""
    rows, I, O = 1100000, 2048, 128
    x = torch.zeros(rows, I, dtype=torch.bfloat16, device="cuda")
    x[-300:] = torch.randn(300, I, device="cuda")
    w = torch.randn(O, I, device="cuda").to(torch.bfloat16) / 32
    out, _ = mem.projection(x, w)
    few = x[-300:].contiguous()
    assert bool((out[:-300] == 0).all())
    want = few.cpu().double() @ w.cpu().double().t()
    near("out", out[-300:], want, sums(few.cpu().double().abs() @ w.cpu().double().abs().t(), I))
    d = torch.zeros(rows, O, dtype=torch.bfloat16, device="cuda")
    d[-300:] = torch.randn(300, O, device="cuda")
    g = mem.projection_backward(d, x, w, float_weight=True)
    last = d[-300:].cpu().double()
    near("gradient of weight", g.weight, last.t() @ few.cpu().double(), sums(last.abs().t() @ few.cpu().double().abs(), 300))
    near("gradient of x", g.x[-300:], last @ w.cpu().double(), sums(last.abs() @ w.cpu().double().abs(), O))
    assert bool((g.x[:-300] == 0).all())


# ---- dropout -----------------------------------------------------------------------------------------------------

DROP_CASES = [
    # dtype, T, n, channels, p, residual, order
    ("f32", 1, 1, 1, 0.5, None, "time"),
    ("bf16", 1, 5, 70, 0.1, "same", "time"),
    ("f16", 3, 4, 64, 0.25, "f32", "slice"),
    ("bf16", 7, 3, 33, 0.5, "f32", "batch"),
    ("f32", 5, 6, 7, 0.1, "same", "batch"),
    ("f32", 4, 9, 130, 0.9, None, "slice"),
    ("bf16", 2, 3, 16, 1.0, "same", "time"),
    ("f16", 2, 3, 17, 0.0, "same", "time"),
    ("f16", 2, 3, 24, 1.0 - 2.0 ** -16, None, "time"),
]


@pytest.mark.parametrize("case", DROP_CASES, ids=case_id)
def test_dropout_and_its_gradient(mem, case):
    dtype, T, n, D, p, residual, order = case
    src = Source(T * 1000 + D, TYPES[dtype], order)
    wide = {None: None, "same": TYPES[dtype], "f32": torch.float32}[residual]
    x, res = src.seq(T, n, D), None if wide is None else src.normal(T, n, D, dtype=wide)
    seed, step, env = 0xFEDCBA9876543210 + D, 2 ** 32 - 2, 2 ** 32 - n if D == 70 else 2 ** 31 - 1
    keep, scale = ref.keep_mask(seed, step, env, T, n, D, p)
    want = ref.dropout(x, keep, scale, res)
    slack = 3 * 2.0 ** -24 * (x.abs() * scale + (0 if res is None else res.abs()))
    got = mem.residual_dropout(src.gpu(x), p, seed, residual=src.gpu(res, wide), step=step, env=env)
    assert got.dtype == (wide or TYPES[dtype])
    near("out", got, want, slack)
    dout = src.normal(T, n, D, dtype=wide or TYPES[dtype])
    back = mem.residual_dropout_backward(src.gpu(dout, wide or TYPES[dtype]), p, seed, step=step, env=env, dtype=TYPES[dtype])
    assert back.dtype == TYPES[dtype] and torch.equal(back.cpu() == 0, ~(keep & (dout * scale != 0)))
    near("gradient of x", back, ref.dropout(dout, keep, scale), 3 * 2.0 ** -24 * dout.abs() * scale)


def test_dropout_masks_of_tokens_are_those_of_the_rollout(mem):
    """Step by step, from the middle of the environments, and with the step's number on the GPU."""
    T, n, D, seed, p = 6, 11, 50, 5, 0.3
    x = torch.randn(T, n, D, device="cuda")
    whole = mem.residual_dropout(x, p, seed, step=2 ** 40 - 3, env=9)
    number = torch.full((1,), 2 ** 40 - 3, dtype=torch.int64, device="cuda")
    for t in range(T):
        assert torch.equal(mem.residual_dropout(x[t], p, seed, step=2 ** 40 - 3 + t, env=9), whole[t])
        assert torch.equal(mem.residual_dropout(x[t, 4:], p, seed, step=2 ** 40 - 3 + t, env=13), whole[t, 4:])
        assert torch.equal(mem.residual_dropout(x[t], p, seed, step=number, env=9), whole[t])
        number += 1
    assert not torch.equal(mem.residual_dropout(x, p, seed + 1, step=2 ** 40 - 3, env=9), whole)


def test_dropout_keeps_its_share_and_its_mean(mem):
    """8.4 million numbers: the share that is kept within five standard deviations; neighbours of step, environment and channel as often alike as chance has it."""
    x = torch.ones(32, 512, 512, device="cuda")
    for p in (0.1, 0.5):
        kept = mem.residual_dropout(x, p, 77) != 0
        n, q = kept.numel(), 1 - p
        assert abs(float(kept.double().mean()) - q) <= 5 * math.sqrt(p * q / n) + 2.0 ** -17
        alike = p * p + q * q
        for a, b in ((kept[1:], kept[:-1]), (kept[:, 1:], kept[:, :-1]), (kept[..., 1:], kept[..., :-1])):
            assert abs(float((a == b).double().mean()) - alike) <= 6 * math.sqrt(alike * (1 - alike) / a.numel()) + 2.0 ** -16


def test_dropout_forgets_what_it_drops(mem):
    """Infinities and NaN in dropped places leave the residual as it is."""
    x, res = torch.full((3, 40), float("nan"), device="cuda"), torch.randn(3, 40, device="cuda")
    out = mem.residual_dropout(x, 0.5, 3, residual=res)
    dropped = ~out.isnan()
    assert 20 < int(dropped.sum()) < 100 and torch.equal(out[dropped], res[dropped])
    assert torch.equal(mem.residual_dropout(x, 1.0, 3, residual=res), res)


# ---- together --------------------------------------------------------------------------------------------------------

def _block(mem, g, p, first, step, state, tail, drop=0.2):
    """One policy block on the residual stream: (residual, state, tail)."""
    token = g.dim() == 2
    inner = p["w_in"].shape[0] // 4
    mixed = mem.projection(g, p["w_in"], p["b_in"])[0] if token else mem.project(g, p["w_in"], p["b_in"])
    x, decay, intake, z = mixed.split(inner, -1)
    if token:
        x, tail = mem.causal_conv_step(x, p["conv"], None, tail, first=first, out_state=torch.empty_like(tail))
        y, state = mem.gated_recurrence_step(x, decay, intake, p["rate"], state, z=z, first=first, out_state=torch.empty_like(state))
        y, _ = mem.projection(y, p["w_out"])
        return mem.residual_dropout(y, drop, 17, residual=g, step=step), state, tail
    x, tail = mem.conv(x, p["conv"], state=tail, first=first)
    y, state = mem.recurrence(x, decay, intake, p["rate"], z=z, state=state, first=first)
    return mem.dropout(mem.project(y, p["w_out"]), drop, 17, residual=g, step=step), state, tail


def _block_parameters(src, width, inner, dtype=torch.float32):
    return {"w_in": src.normal(4 * inner, width, spread=width ** -0.5).to("cuda", dtype), "b_in": plain(src.normal(4 * inner)), "conv": plain(src.normal(inner, 4)),
            "rate": plain(-torch.exp(src.normal(inner) - 1.0)), "w_out": src.normal(width, inner, spread=inner ** -0.5).to("cuda", dtype)}


def test_a_block_acts_as_it_learns(mem):
    """Token by token and as a rollout, the same block gives the same stream, masks and all; then its gradients against 64 bits.  About six sums
    of up to 200 terms follow one another: 12 * 32 * 2^-24 * sqrt(200) = 3.3e-4 of the largest value."""
    src = Source(91, torch.float32)
    T, n, width, inner = 20, 7, 72, 50
    p, g, first = _block_parameters(src, width, inner), plain(src.seq(T, n, width)), src.flags(T, n, 0.1).cuda()
    state, tail = plain(src.normal(n, inner)), plain(src.normal(n, 3, inner))
    whole, last, last_tail = _block(mem, g, p, first, 1000, state, tail)
    s, c = state, tail
    for t in range(T):
        out, s, c = _block(mem, g[t], p, first[t], 1000 + t, s, c)
        assert float((out - whole[t]).abs().max()) <= 3.3e-4 * float(whole.abs().max()), t
    assert float((s - last).abs().max()) <= 3.3e-4 * float(last.abs().max())

    import memory_reference as older
    keep, scale = ref.keep_mask(17, 1000, 0, T, n, width, 0.2)
    leaf = {k: v.cpu().double().requires_grad_(True) for k, v in {**p, "g": g, "state": state, "tail": tail}.items()}
    x, decay, intake, z = ref.project(leaf["g"], leaf["w_in"], leaf["b_in"])[0].split(inner, -1)
    x, _ = older.conv(x, leaf["conv"], state=leaf["tail"], first=first.cpu())
    y, h = ref.recurrence(x, decay, intake, leaf["rate"], z=z, state=leaf["state"], first=first.cpu())
    out = ref.dropout(ref.project(y, leaf["w_out"])[0], keep, scale, leaf["g"])
    w, wh = src.seq(T, n, width), src.normal(n, inner)
    ((out * w).sum() + (h * wh).sum()).backward()
    mine = {k: v.detach().clone().requires_grad_(True) for k, v in {**p, "g": g, "state": state, "tail": tail}.items()}
    got, got_h, _ = _block(mem, mine["g"], mine, first, 1000, mine["state"], mine["tail"])
    ((got * plain(w)).sum() + (got_h * plain(wh)).sum()).backward()
    assert float((got.detach().cpu().double() - out.detach()).abs().max()) <= 3.3e-4 * float(out.detach().abs().max())
    for k in leaf:
        big = float(leaf[k].grad.abs().max())
        assert float((mine[k].grad.cpu().double() - leaf[k].grad).abs().max()) <= 3.3e-4 * big, k


def test_a_projection_of_16_bits_takes_float32_parameters(mem):
    """weight float32, activations bfloat16: the product of the rounded weight, a float32 gradient."""
    src = Source(93, torch.bfloat16)
    x, w, b = src.seq(4, 30, 64), src.normal(48, 64, spread=0.125), src.normal(48)
    gx, gw, gb = src.gpu(x).requires_grad_(True), plain(w).requires_grad_(True), plain(b).requires_grad_(True)
    res = plain(src.normal(4, 30, 48)).requires_grad_(True)
    out = mem.project(gx, gw, gb, residual=res, act="silu")
    want, pre = mem.projection(src.gpu(x), plain(w).bfloat16(), plain(b), residual=res.detach(), act="silu", save=True)
    assert torch.equal(out, want) and out.dtype == torch.float32
    d = plain(src.normal(4, 30, 48))
    out.backward(d)
    g = mem.projection_backward(d, src.gpu(x), plain(w).bfloat16(), plain(b), pre=pre, act="silu", float_weight=True)
    assert gw.grad.dtype == torch.float32 and torch.equal(gw.grad, g.weight) and torch.equal(gx.grad, g.x) and torch.equal(gb.grad, g.bias) and torch.equal(res.grad, d)
    # a sum over the output hands over an expanded gradient
    for leaf in (gx, gw, gb, res):
        leaf.grad = None
    mem.project(gx, gw, gb, residual=res).sum().backward()
    assert bool((res.grad == 1).all()) and torch.allclose(gb.grad, torch.full_like(gb, 120.0))
    with torch.no_grad():
        assert not mem.project(gx, gw, gb, act="silu").requires_grad


def _all_operators(mem, g, w, first, number):
    out, pre = mem.projection(g["x"], w["in"], w["bias"], act="gelu_tanh", save=True)
    x, decay, intake = out.split(out.shape[-1] // 3, -1)
    y, h, saved = mem.gated_recurrence(x, decay, intake, w["rate"], z=x, state=g["state"], first=first, save=True)
    back, _ = mem.projection(y, w["out"], residual=g["x"])
    drop = mem.residual_dropout(back, 0.3, 5, residual=g["x"], step=number)
    dd = mem.residual_dropout_backward(drop, 0.3, 5, step=number)
    db = mem.projection_backward(dd, y, w["out"])
    dr = mem.gated_recurrence_backward(db.x, saved, x, decay, intake, w["rate"], z=x, state=g["state"], first=first)
    dp = mem.projection_backward(torch.cat([dr.x, dr.decay, dr.intake], -1), g["x"], w["in"], w["bias"], pre=pre, act="gelu_tanh")
    return [v for v in (out, pre, y, h, back, drop, dd, *db, *dr, *dp) if v is not None]


@pytest.mark.parametrize("T,n,width,inner", [(150, 2, 96, 64), (40, 130, 72, 88)])
def test_operators_on_another_stream_and_in_a_graph(mem, T, n, width, inner):
    """On a side stream, and captured once and replayed with other inputs and another step's number in the same tensors: bit for bit as eager."""
    src = Source(51, torch.bfloat16)
    w = {"in": src.gpu(src.normal(3 * inner, width, spread=0.1)), "bias": plain(src.normal(3 * inner)), "rate": plain(-torch.exp(src.normal(inner))),
         "out": src.gpu(src.normal(width, inner, spread=0.1))}
    sets = [{"x": src.gpu(src.seq(T, n, width)), "state": plain(src.normal(n, inner))} for _ in range(3)]
    first = src.flags(T, n, 0.05).cuda()
    numbers = [torch.full((1,), 1000 * k, dtype=torch.int64, device="cuda") for k in range(3)]
    want = [[v.clone() for v in _all_operators(mem, s, w, first, k)] for s, k in zip(sets, numbers)]
    again = _all_operators(mem, sets[1], w, first, numbers[1])
    assert all(torch.equal(a, b) for a, b in zip(again, want[1]))
    assert not torch.equal(_all_operators(mem, sets[1], w, first, numbers[2])[5], want[1][5])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _all_operators(mem, sets[0], w, first, numbers[0])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    held, number = {k: v.clone() for k, v in sets[0].items()}, numbers[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all_operators(mem, held, w, first, number)
    for k in (1, 2, 0, 1):
        for name in held:
            held[name].copy_(sets[k][name])
        number.copy_(numbers[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[k])), k
        mem.projection(sets[0]["x"], w["in"])
        torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 8, 40, 2000])
@pytest.mark.parametrize("D", [66, 3])
def test_recurrence_updates_a_state_in_place(mem, T, D):
    """At the C entry state_out may be state_in, for one part of steps as for many."""
    from paper_2402_16801_amd import binding as cx
    lib, n = cx.load(), 2
    x, decay, intake, y = (torch.randn(T, n, D, device="cuda") for _ in range(4))
    rate, state = -torch.rand(D, device="cuda") * 0.01, torch.randn(n, D, device="cuda")
    want_y, want, _ = mem.gated_recurrence(x, decay, intake, rate, state=state)
    views = {f: v for k, t in (("x", x), ("decay", decay), ("intake", intake), ("y", y)) for f, v in ((k, t.data_ptr()), (k + "_step", n * D), (k + "_env", D))}
    args = cx.RecurrenceArgs(dtype=0, steps=T, n=n, channels=D, rate=rate.data_ptr(), state_in=state.data_ptr(), state_out=state.data_ptr(), **views)
    need = lib.craftax_gated_recurrence_workspace_bytes(args, 0)
    work = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    args.workspace, args.workspace_bytes = work.data_ptr(), need
    torch.cuda.synchronize()
    assert lib.craftax_gated_recurrence(args, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(y, want_y) and torch.equal(state, want)


@pytest.mark.parametrize("size", [(40, 130, 72, 88), (150, 2, 96, 64)])
def test_calls_on_two_streams_at_once(mem, size):
    """Each call has its own workspace: two streams that work at the same time give what they give alone, again and again."""
    T, n, width, inner = size
    src = Source(53, torch.bfloat16)
    w = {"in": src.gpu(src.normal(3 * inner, width, spread=0.1)), "bias": plain(src.normal(3 * inner)), "rate": plain(-torch.exp(src.normal(inner))),
         "out": src.gpu(src.normal(width, inner, spread=0.1))}
    sets = [{"x": src.gpu(src.seq(T, n, width)), "state": plain(src.normal(n, inner))} for _ in range(2)]
    first = src.flags(T, n, 0.05).cuda()
    number = torch.zeros(1, dtype=torch.int64, device="cuda")
    want = [[v.clone() for v in _all_operators(mem, s, w, first, number)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        got = []
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append(_all_operators(mem, s, w, first, number))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, v in zip(got, want) for a, b in zip(g, v))


def test_states_of_the_recurrence_as_autograd_sees_them(mem):
    from paper_2402_16801_amd import binding
    src = Source(97, torch.float32)
    args, how = rec_args(rec_gpu(src, rec_inputs(src, 5, 3, 20, True, True)))
    token = [a if a.dim() == 1 else a[0] for a in args]
    state = how["state"]
    leaf = args[0].clone().requires_grad_(True)
    y, h = mem.recurrence(leaf, *args[1:], **how)
    (want,) = torch.autograd.grad(y.sum() + h.sum(), leaf, retain_graph=True)
    version = state._version
    assert mem.gated_recurrence_step(*token, state)[1] is state and state._version == version + 1
    (same,) = torch.autograd.grad(y.sum() + h.sum(), leaf)           # the state's values are kept apart
    assert torch.equal(same, want)
    grown = state.clone().requires_grad_(True)
    with pytest.raises(binding.CraftaxError, match="requires gradients"):
        mem.gated_recurrence_step(*token, grown)
    with torch.no_grad():
        assert mem.gated_recurrence_step(*token, grown)[1] is grown
    y, _ = mem.recurrence(*args, **how)
    assert not y.requires_grad
    (g,) = torch.autograd.grad(mem.recurrence(*args, z=how["z"], state=grown)[0].sum(), grown)
    assert g.shape == grown.shape
    x = args[0].clone().requires_grad_(True)
    number = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = mem.dropout(x, 0.5, 1, step=number)
    number += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


# ---- refusals ------------------------------------------------------------------------------------------------------------

def test_refusals(mem):
    from paper_2402_16801_amd import binding
    src = Source(81, torch.float32)
    g = rec_gpu(src, rec_inputs(src, 4, 3, 32, True, True))
    args, how = rec_args(g)
    x = g["x"]

    def refused(text, call, *a, **k):
        with pytest.raises(binding.CraftaxError, match=text):
            call(*a, **k)

    refused("no CPU path", mem.gated_recurrence, x.cpu(), *args[1:])
    refused("float32, bfloat16 or float16", mem.gated_recurrence, x.double(), *args[1:])
    refused("decay has shape", mem.gated_recurrence, x, args[1][:3], *args[2:])
    refused("intake is", mem.gated_recurrence, x, args[1], args[2].half(), args[3])
    refused("rate has shape", mem.gated_recurrence, *args[:3], args[3][:31])
    refused("state", mem.gated_recurrence, *args, state=torch.zeros(3, 31, device="cuda"))
    refused("lengths", mem.gated_recurrence, *args, lengths=torch.zeros(3, dtype=torch.int64, device="cuda"))
    refused("first must be", mem.gated_recurrence, *args, first=torch.zeros(4, 3, device="cuda"))
    refused("steps, n and channels must be positive", mem.gated_recurrence, *[a[:0] for a in args[:3]], args[3])
    refused("saved is not", mem.gated_recurrence_backward, x, None, *args)
    refused("saved is not", mem.gated_recurrence_backward, x, torch.zeros(8, dtype=torch.uint8, device="cuda"), *args)
    w = torch.zeros(16, 32, device="cuda")
    refused("no CPU path", mem.projection, x.cpu(), w)
    refused("weight is", mem.projection, x, w.half())
    refused("weight has shape", mem.projection, x, w[:, :31])
    refused("weight must be", mem.projection, x, w[0])
    refused("side by side", mem.projection, x, torch.zeros(16, 2, 32, 2, device="cuda")[:, 0, :, 0])
    refused("side by side", mem.projection, x.transpose(1, 2).contiguous().transpose(1, 2), w)
    refused("bias has shape", mem.projection, x, w, torch.zeros(15, device="cuda"))
    refused("residual must be", mem.projection, x, w, residual=torch.zeros(4, 3, 16, dtype=torch.float16, device="cuda"))
    refused("residual has shape", mem.projection, x, w, residual=torch.zeros(4, 3, 15, device="cuda"))
    refused("act must be", mem.projection, x, w, act="tanh")
    refused("must be positive", mem.projection, x[:0], w)
    refused("must be positive", mem.projection, x, w[:0])
    refused("must be positive", mem.projection, x[..., :0], w[:, :0])
    d = torch.zeros(4, 3, 16, device="cuda")
    refused("pre is NULL", mem.projection_backward, d, x, w, act="silu")
    refused("dout has shape", mem.projection_backward, d[:3], x, w)
    refused("dout must be", mem.projection_backward, d.half(), x, w)
    refused("p must be 0..1", mem.residual_dropout, x, 1.5, 1)
    refused("p must be 0..1", mem.residual_dropout, x, float("nan"), 1)
    refused("seed must be", mem.residual_dropout, x, 0.5, -1)
    refused("seed must be", mem.residual_dropout, x, 0.5, 2 ** 64)
    refused("step must be a whole", mem.residual_dropout, x, 0.5, 1, step=2 ** 63)
    refused("step \\+ steps", mem.residual_dropout, x, 0.5, 1, step=-1)
    refused("step \\+ steps", mem.residual_dropout, x, 0.5, 1, step=2 ** 63 - 4)
    refused("env \\+ n", mem.residual_dropout, x, 0.5, 1, env=2 ** 32 - 2)
    refused("env \\+ n", mem.residual_dropout, x, 0.5, 1, env=-1)
    refused("step is", mem.residual_dropout, x, 0.5, 1, step=torch.zeros(1, device="cuda"))
    refused("one number", mem.residual_dropout, x, 0.5, 1, step=torch.zeros(2, dtype=torch.int64, device="cuda"))
    refused("must be positive", mem.residual_dropout, x[:0], 0.5, 1)
    refused("must be float32, bfloat16", mem.residual_dropout_backward, x, 0.5, 1, dtype=torch.float64)
    refused("out_dtype", mem.residual_dropout_backward, x.half(), 0.5, 1, dtype=torch.bfloat16)
    refused("residual must be", mem.residual_dropout, x, 0.5, 1, residual=x.half())
    torch.cuda.synchronize()


def test_refusals_at_the_c_entry(mem):
    """Codes and texts of the calls themselves; nothing is launched."""
    from paper_2402_16801_amd import binding as cx
    lib = cx.load()
    for name in ("gated_recurrence", "gated_recurrence_backward", "projection", "projection_backward", "residual_dropout"):
        assert getattr(lib, "craftax_" + name)(None, None) == -1
    v = torch.zeros(4096, device="cuda")
    p = v.data_ptr()

    def codes(call, good, cases):
        for field, value, code in cases:
            bad = type(good).from_buffer_copy(good)
            setattr(bad, field, value)
            assert call(bad, None) == code, (field, value)
            assert lib.craftax_last_error()

    rec = cx.RecurrenceArgs(dtype=0, steps=1, n=1, channels=4, rate=p, x=p, decay=p, intake=p, y=p + 64)
    assert lib.craftax_gated_recurrence(rec, None) == 0
    codes(lib.craftax_gated_recurrence, rec, (("dtype", 3, -6), ("steps", 0, -3), ("n", -1, -3), ("channels", 2 ** 31 - 4095, -3), ("rate", None, -1), ("x", p + 2, -2),
                                              ("y", None, -1), ("saved", p + 16, -2), ("state_in", p + 1, -2)))
    rec.saved, rec.dy, rec.dx, rec.ddecay, rec.dintake, rec.drate = p, p, p + 64, p + 128, p + 192, p + 256
    need = lib.craftax_gated_recurrence_workspace_bytes(rec, 1)
    assert need > 0 and lib.craftax_gated_recurrence_backward(rec, None) == -1
    rec.workspace, rec.workspace_bytes = p + 4096, need - 1
    assert lib.craftax_gated_recurrence_backward(rec, None) == -3
    rec.workspace, rec.workspace_bytes = p + 4100, need
    assert lib.craftax_gated_recurrence_backward(rec, None) == -2
    rec.z = p
    assert lib.craftax_gated_recurrence_backward(rec, None) == -1 and b"dz" in lib.craftax_last_error()
    assert lib.craftax_gated_recurrence_saved_bytes(cx.RecurrenceArgs()) == 0 and lib.craftax_gated_recurrence_workspace_bytes(cx.RecurrenceArgs(), 1) == 0
    pro = cx.ProjectionArgs(dtype=0, out_dtype=0, steps=1, n=1, inputs=4, outputs=4, weight=p, weight_row=4, weight_column=1, x=p, out=p + 256)
    assert lib.craftax_projection(pro, None) == 0
    codes(lib.craftax_projection, pro, (("dtype", 3, -6), ("out_dtype", 1, -6), ("act", 4, -6), ("inputs", 0, -3), ("outputs", 2 ** 31 - 4095, -3), ("weight_column", 2, -3),
                                        ("weight", None, -1), ("out", None, -1), ("x", p + 2, -2), ("bias", p + 1, -2)))
    pro.weight_row, pro.weight_column = 1, 4
    need = lib.craftax_projection_workspace_bytes(pro, 0)
    assert need > 0 and lib.craftax_projection(pro, None) == -1
    pro.workspace, pro.workspace_bytes = p + 4096, need - 1
    assert lib.craftax_projection(pro, None) == -3
    pro.steps, pro.n = 1 << 20, 1 << 11
    assert lib.craftax_projection(pro, None) == -3 and lib.craftax_projection_workspace_bytes(pro, 0) == 0
    pro.steps, pro.n, pro.inputs, pro.outputs = 1, 1 << 25, 1 << 18, 1
    assert lib.craftax_projection(pro, None) == -3 and b"memory" in lib.craftax_last_error()
    assert lib.craftax_projection_backward(pro, None) == -3
    drop = cx.DropoutArgs(dtype=0, out_dtype=0, steps=1, n=1, channels=4, p=0.5, x=p, out=p + 64)
    assert lib.craftax_residual_dropout(drop, None) == 0
    codes(lib.craftax_residual_dropout, drop, (("dtype", 3, -6), ("out_dtype", 3, -6), ("p", -0.1, -6), ("steps", 0, -3), ("channels", 0, -3), ("step", -1, -3),
                                               ("env", 2 ** 32, -3), ("x", None, -1), ("out", p + 2, -2), ("step_at", p + 4, -2)))
    torch.cuda.synchronize()


def test_everything_on_the_tensors_own_device_and_nothing_else(mem):
    """Tensors of one call on two devices are refused before anything runs."""
    from paper_2402_16801_amd import binding
    x, w = torch.zeros(2, 3, 8, device="cuda"), torch.zeros(8)
    for call in (lambda: mem.gated_recurrence(x, x, x, w), lambda: mem.projection(x, torch.zeros(4, 8)), lambda: mem.residual_dropout(x, 0.5, 1, residual=x.cpu()),
                 lambda: mem.residual_dropout(x, 0.5, 1, step=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(binding.CraftaxError, match="cpu"):
            call()
