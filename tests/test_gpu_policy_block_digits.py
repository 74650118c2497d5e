"""The digits that the gated recurrence, the projection and the norm's gate keep where numbers are far from 1: gates that are nearly open, activations
beyond the range of their type, small and large gradients, parts of float32 values.  Tolerances are relative and derived beside each test."""
import pytest
import torch

import policy_block_reference as ref
from test_gpu_memory import ROUND, TYPES, Source, plain
from test_gpu_policy_block import near, sums

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mem():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2402_16801_amd import memory
    return memory


def relative(what, got, want, allowed):
    """Every value, however small, off by no more than that share of itself."""
    got64 = got.detach().cpu().double()
    assert got64.shape == want.shape, (what, got64.shape, want.shape)
    off = ((got64 - want).abs() / want.abs())
    assert bool((off <= allowed).all()), f"{what}: off by {float(off.max()):.3g} of a value, {allowed:.3g} are allowed"


# ---- float32 gradients of float16 activations --------------------------------------------------------------------

GRADIENT_CASES = [
    # rows, inputs, outputs, act: fragments, heads, tiles through registers, straight to LDS, in parts
    (5, 40, 30, "none"),
    (64, 1345, 18, "silu"),
    (700, 300, 400, "gelu_tanh"),
    (3000, 72, 44, "relu"),
    (33000, 128, 136, "none"),
    (20000, 512, 264, "silu"),
]


@pytest.mark.parametrize("size", [2.0 ** -30, 2.0 ** 24, 2.0 ** -140], ids=["small", "large", "smallest"])
@pytest.mark.parametrize("case", GRADIENT_CASES, ids=str)
def test_projection_of_float16_takes_float32_gradients_of_any_size(mem, case, size):
    """dp comes to the matrix units in float16: values above 65,504 and below 6e-8 have to get there.  Rounded relative to itself, 2^-11, as long as
    it is above 2^-29 of the largest; rows are up to 2^-20 apart here.  Gradients of the weight are compared in units of `size`, an exact scaling; those of
    x have 16 bits (near's 2^-25 is half of their smallest step).  The smallest: float32 numbers below the normal ones, whole multiples of 2^-149, so that
    dp has 2^-150 more, 2^-10 in units of `size`, and what is computed of them 2^-149 on top."""
    rows, I, O, act = case
    src = Source(rows + I, torch.float16)
    x, w = src.seq(1, rows, I)[0], src.normal(O, I, spread={2.0 ** -30: 2.0 ** 10, 2.0 ** 24: 2.0 ** -20, 2.0 ** -140: 2.0 ** 10}[size], dtype=torch.float16)
    dout = (src.normal(rows, O) * size).float().double()
    dout[rows // 2] = (dout[rows // 2] * 2.0 ** -20).float().double() if size > 2.0 ** -100 else 0.0
    pre = src.normal(rows, O, spread=2.0, dtype=torch.float16)
    given = pre.clone().requires_grad_(True)
    (dp,) = torch.autograd.grad(ref.act(given, act), given, dout)
    step = 2.0 ** -9 if size < 2.0 ** -100 else 0.0
    g = mem.projection_backward(plain(dout), src.gpu(x), src.gpu(w), torch.zeros(O, device="cuda"), pre=None if act == "none" else src.gpu(pre), act=act,
                                float_weight=True)
    off = 1.1 * ROUND[torch.float16] + 2.0 ** -21
    terms = dp.abs().t() @ x.abs()
    near("gradient of weight", (g.weight.double() / size).float(), (dp.t() @ x) / size, (terms * off + sums(terms, rows)) / size + step * x.abs().sum(0))
    near("gradient of bias", (g.bias.double() / size).float(), dp.sum(0) / size, (dp.abs().sum(0) * 2.0 ** -21 + sums(dp.abs().sum(0), rows)) / size + step * rows)
    terms = dp.abs() @ w.abs()
    near("gradient of x", g.x, dp @ w, terms * off + sums(terms, O))
    assert size < 2.0 ** -100 or bool((g.weight != 0).any(1).all())


@pytest.mark.parametrize("case", GRADIENT_CASES, ids=str)
def test_projection_of_float16_keeps_infinite_gradients_in_their_rows(mem, case):
    """Infinities and NaN among float32 gradients stay in their row of dx, whatever the others' size; gradients that are all 0 give 0."""
    rows, I, O, act = case
    src = Source(rows, torch.float16)
    x, w, pre = src.seq(1, rows, I)[0], src.normal(O, I, spread=2.0 ** 10, dtype=torch.float16), src.normal(rows, O, dtype=torch.float16)
    dout = (src.normal(rows, O) * 2.0 ** -30).float().double()
    spoilt = dout.clone()
    spoilt[1, 0], spoilt[rows - 1, O - 1] = float("inf"), float("nan")
    how = {"pre": None if act == "none" else src.gpu(pre).abs(), "act": act, "float_weight": True}
    given = pre.abs().requires_grad_(True)
    (dp,) = torch.autograd.grad(ref.act(given, act), given, dout)
    g = mem.projection_backward(plain(spoilt), src.gpu(x), src.gpu(w), None, **how)
    fine = [m for m in range(rows) if m not in (1, rows - 1)]
    terms = dp[fine].abs() @ w.abs()
    near("gradient of x", g.x[fine], dp[fine] @ w, terms * (1.1 * ROUND[torch.float16] + 2.0 ** -21) + sums(terms, O))
    assert not bool(torch.isfinite(g.x[1]).any()) and bool(g.x[rows - 1].isnan().all())
    g = mem.projection_backward(torch.zeros(rows, O, device="cuda"), src.gpu(x), src.gpu(w), torch.zeros(O, device="cuda"), **how)
    assert all(bool((v == 0).all()) for v in g)


@pytest.mark.parametrize("O", [2200001, 1100000])
def test_projection_of_float16_finds_the_size_of_its_gradients_in_many_columns(mem, O):
    """More columns than blocks lie side by side for: the largest value is in the last ones, and scaled as if it were not it would be infinite."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w = (torch.randint(-2, 3, shape, generator=gen, device="cuda").half() for shape in ((3, 8), (O, 8)))
    dout = torch.zeros(3, O, device="cuda")
    dout[:, :5] = 2.0 ** 10
    dout[:, -3:] = 2.0 ** 20 * torch.randint(1, 4, (3, 3), generator=gen, device="cuda").float()
    g = mem.projection_backward(dout, x, w, torch.zeros(O, device="cuda"), float_weight=True)
    assert torch.equal(g.weight.double(), dout.double().t() @ x.double()) and torch.equal(g.bias.double(), dout.double().sum(0))
    assert torch.equal(g.x, (dout.double() @ w.double()).half())


def test_projection_of_float16_finds_the_size_of_its_gradients_at_every_replay(mem):
    """Captured once, replayed with gradients of other sizes in the same tensor, on a side stream beside eager calls: bit for bit as eager."""
    src = Source(5, torch.float16)
    x, w, pre = src.gpu(src.normal(3000, 72, dtype=torch.float16)), src.gpu(src.normal(136, 72, dtype=torch.float16)), src.gpu(src.normal(3000, 136, dtype=torch.float16))
    douts = [plain(src.normal(3000, 136) * size) for size in (1.0, 2.0 ** -40, 2.0 ** 30, 0.0, 2.0 ** -20)]
    bias = torch.zeros(136, device="cuda")

    def back(dout):
        return mem.projection_backward(dout, x, w, bias, pre=pre, act="silu", float_weight=True)

    want = [[v.clone() for v in back(d)] for d in douts]
    given, side, graph = douts[0].clone(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        back(given)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = back(given)
    for turn in range(2):
        for d, exp in zip(douts, want):
            given.copy_(d)
            graph.replay()
            eager = back(douts[turn + 1])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, exp))
            assert all(torch.equal(a, b) for a, b in zip(eager, want[turn + 1]))


# ---- activations beyond the range of their type ---------------------------------------------------------------------

def test_slopes_of_infinite_arguments_are_0_and_1(mem):
    """pre in 16 bits may be an infinity where the sum was not."""
    for dtype in TYPES.values():
        most = torch.finfo(dtype).max
        pre = torch.tensor([[-float("inf"), -most, -most / 8, most / 8, most, float("inf"), float("nan")]], dtype=dtype, device="cuda")
        for act in ("relu", "silu", "gelu_tanh"):
            g = mem.projection_backward(torch.ones(1, 7, dtype=dtype, device="cuda"), torch.ones(1, 1, dtype=dtype, device="cuda"),
                                        torch.ones(7, 1, dtype=dtype, device="cuda"), torch.zeros(7, device="cuda"), pre=pre, act=act, want_x=False)
            for got in (g.weight[:, 0].float(), g.bias):
                assert got[:6].tolist() == [0.0, 0.0, 0.0, 1.0, 1.0, 1.0] and bool(got[6].isnan()), (act, dtype, got)


@pytest.mark.parametrize("act", ["relu", "silu", "gelu_tanh"])
def test_projection_beyond_the_range_of_float16(mem, act):
    """Sums of 160,000 on a float32 residual: out holds them, pre does not, and the backward pass has their slope."""
    x = torch.full((40, 64), 50.0, dtype=torch.float16, device="cuda")
    x[::2] = -50.0
    w = torch.full((24, 64), 50.0, dtype=torch.float16, device="cuda")
    out, pre = mem.projection(x, w, residual=torch.ones(40, 24, device="cuda"), act=act, save=True)
    assert bool((out[1::2] == 160001.0).all()) and bool((out[::2] == 1.0).all()) and bool(pre.isinf().all())
    g = mem.projection_backward(torch.ones(40, 24, device="cuda"), x, w, torch.zeros(24, device="cuda"), pre=pre, act=act, float_weight=True)
    assert bool((g.x[1::2] == 1200.0).all()) and bool((g.x[::2] == 0.0).all())
    assert bool((g.weight == 1000.0).all()) and bool((g.bias == 20.0).all())


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_slopes_keep_their_digits(mem, act):
    """A slope is a product of at most eight factors and sums of size 1.2 or less, each rounded once to 2^-24, and an exponential whose argument, at most
    3 where it counts for that much, is rounded to 2^-23: 2^-20 in all."""
    pre = torch.linspace(-20.0, 20.0, 40001).double().float()
    given = pre.double().requires_grad_(True)
    (want,) = torch.autograd.grad(ref.act(given, act).sum(), given)
    g = mem.projection_backward(torch.ones(1, 40001, device="cuda"), torch.ones(1, 1, device="cuda"), torch.ones(40001, 1, device="cuda"),
                                torch.zeros(40001, device="cuda"), pre=pre.cuda()[None], act=act, want_x=False)
    off = (g.bias.cpu().double() - want).abs()
    assert float(off.max()) <= 2.0 ** -20, (float(off.max()), float(pre[off.argmax()]))


# ---- gates that are nearly open -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,D", [(1, 3, 64), (300, 2, 64), (3, 5000, 64)])
def test_recurrence_gradients_of_gates_that_are_nearly_open(mem, dtype, T, n, D):
    """Gates of 10 to 25, value by value.  Every step begins an episode, so that a gradient is a product: dintake = dy m x q (1 - q), ddecay = -dy q x a a / m
    rate s (1 - s).  1 - q is an exponential whose argument, up to 36 in units of the base's, is rounded to 2^-19 and has a constant right to 2^-25 of it:
    2.1e-6.  Some 16 factors and roundings of 2^-23 are 1.9e-6, together below 2^-17."""
    src = Source(T + n, TYPES[dtype])
    decay, intake = (10.0 + 15.0 * torch.rand(T, n, D, generator=src.gen) for _ in range(2))
    decay, intake = decay.to(TYPES[dtype]).double(), intake.to(TYPES[dtype]).double()
    x, dy = (src.seq(T, n, D).abs().clamp(min=0.1).to(TYPES[dtype]).double() for _ in range(2))
    rate = (-torch.exp(src.normal(D) - 1.0)).float().double()
    args = [src.gpu(x), src.gpu(decay), src.gpu(intake), plain(rate)]
    first = torch.ones(T, n, dtype=torch.uint8, device="cuda")
    _, _, saved = mem.gated_recurrence(*args, first=first, save=True)
    g = mem.gated_recurrence_backward(src.gpu(dy), saved, *args, first=first)
    s, q = torch.sigmoid(decay), torch.sigmoid(intake)
    log_a = rate * s
    m = torch.sqrt(-torch.expm1(2 * log_a))
    allowed = 2.0 ** -17 + (ROUND[TYPES[dtype]] * (1 + 2.0 ** -8) if dtype != "f32" else 0.0)
    relative("gradient of intake", g.intake, dy * m * x * q * torch.sigmoid(-intake), allowed)
    relative("gradient of decay", g.decay, -dy * q * x * torch.exp(2 * log_a) / m * rate * s * torch.sigmoid(-decay), allowed)
    relative("gradient of x", g.x, dy * m * q, allowed)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("D", [200, 5000])
def test_norm_gradients_of_gates_that_are_nearly_open(mem, dtype, act, D):
    """As for the recurrence's gates, in rows that registers hold and in long ones.  Without a norm after the block and with du = 0 the gradient of the gate is dout y act'(gate)."""
    src = Source(7, TYPES[dtype])
    gate = (10.0 + 15.0 * torch.rand(5, 9, D, generator=src.gen)).to(TYPES[dtype]).double()
    y, dout = (src.seq(5, 9, D).abs().clamp(min=0.1).to(TYPES[dtype]).double() for _ in range(2))
    g = mem.residual_norm_backward(src.gpu(dout), torch.zeros(5, 9, D, dtype=TYPES[dtype], device="cuda"), src.gpu(y), src.gpu(y), gate=src.gpu(gate), gate_act=act)
    rest = torch.sigmoid(-gate)
    slope = torch.sigmoid(gate) * (rest if act == "sigmoid" else 1 + gate * rest)
    relative("gradient of gate", g.gate, dout * y * slope, 2.0 ** -17 + (ROUND[TYPES[dtype]] * (1 + 2.0 ** -8) if dtype != "f32" else 0.0))


# ---- parts of float32 values -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("shift", [0, -110, -120, 100])
def test_projection_of_float32_by_value(mem, shift):
    """Sums of one product, by tiles: every value right to 2^-22 of itself, whatever its last digits.  What the three parts leave out of a product is
    below 2^-24 + 2^-34 of it, an addition of the matrix units may cut off 2^-23, and the smaller products' additions add 2^-30 each.  Values from 2^-110
    on have all of their digits in three parts; smaller ones lose half a step of bfloat16's smallest numbers, 2^-134."""
    src = Source(3, torch.float32)
    allowed = 2.0 ** -22 + (2.0 ** (-134 - shift) if shift < -110 else 0.0)
    bits = torch.tensor([0x3F80FFFF, 0x3FFFFFFF, 0x3F807FFF, 0x3F808000, 0x3F80FF80, 0x3F80807F, 0x3F807F7F, 0x3F808080, 0x3F800001, 0x3FFF7FFF, 0x3FFF8000, 0x3FFF8001],
                        dtype=torch.int32).view(torch.float32).double()

    def some(count):
        v = torch.cat([bits, 1.0 + torch.rand(count, generator=src.gen, dtype=torch.float64) / 128, 1.0 + torch.rand(count, generator=src.gen, dtype=torch.float64)])
        return v[torch.randperm(len(v), generator=src.gen)[:count]].float().double() * (1 - 2 * torch.randint(0, 2, (count,), generator=src.gen))

    x, w = some(700) * 2.0 ** shift, some(400) * 2.0 ** -shift
    x[:12], w[:12] = bits * 2.0 ** shift, bits * 2.0 ** -shift
    out, _ = mem.projection(plain(x)[:, None], plain(w)[:, None])
    relative("out", out, x[:, None] * w[None], allowed)
    # a sum over rows that begins anywhere: the other values are 0
    for k in (0, 5, 69):
        wide, other = torch.zeros(700, 70, dtype=torch.float64), torch.zeros(400, 70, dtype=torch.float64)
        wide[:, k], other[:, k] = x, w
        out, _ = mem.projection(plain(wide), plain(other))
        relative("out", out, x[:, None] * w[None], allowed)
    d = torch.zeros(90, 400, dtype=torch.float64)
    d[17] = w
    wide = torch.zeros(90, 700, dtype=torch.float64)
    wide[17] = x
    g = mem.projection_backward(plain(d), plain(wide), torch.zeros(400, 700, device="cuda"), want_x=False)
    relative("gradient of weight", g.weight, w[:, None] * x[None], allowed)


def test_projection_of_float32_next_to_the_largest_number(mem):
    """Numbers that bfloat16 would round to infinity."""
    most = torch.finfo(torch.float32).max
    x = torch.ones(700, 40, dtype=torch.float64)
    w = torch.ones(400, 40, dtype=torch.float64)
    x[5], x[6] = 0.0, 0.0
    x[5, 3], x[6, 39] = most, -most
    w[:, 3] = w[:, 39] = 2.0 ** -20
    out, _ = mem.projection(plain(x), plain(w))
    relative("out", out, x @ w.t(), 2.0 ** -20)


# ---- states that grow ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,n", [(2000, 1), (2000, 3), (300, 1), (40, 3000)])
def test_recurrence_of_nothing_is_nothing_whatever_its_rate(mem, T, n):
    """Rates above 0, where the root counts as 0: a state of 0 stays 0 however large the product of the factors becomes, and so does a gradient of 0.  One
    that begins at 1e-30 grows alike in one walk and in parts, as long as it is a number (a sum of T logarithms of factors, each off by 2^-22: 2^-11 for T = 2,000)."""
    src = Source(T, torch.float32)
    D = 70
    t = {k: src.normal(T, n, D) for k in ("x", "decay", "intake", "z")}
    rate = torch.full((D,), 2.0)
    rate[::2] = -2.0
    args, z = [plain(t[k]) for k in ("x", "decay", "intake")] + [rate.cuda()], plain(t["z"])
    y, h, saved = mem.gated_recurrence(*args, z=z, save=True)
    assert bool(torch.isfinite(y).all()) and bool((y[..., 1::2] == 0).all()) and bool((h[:, 1::2] == 0).all()) and bool((h[:, ::2] != 0).all())
    g = mem.gated_recurrence_backward(torch.zeros_like(y), saved, *args, z=z, state=torch.zeros_like(h), dstate=torch.zeros_like(h))
    assert all(bool((v == 0).all()) for v in g)
    state = torch.full((n, D), 1e-30, device="cuda")
    y, h, _ = mem.gated_recurrence(*args, state=state)
    log = torch.cumsum(2.0 * torch.sigmoid(t["decay"][..., 1::2]), 0)
    want = 1e-30 * torch.exp(log)
    number = want < 1e38
    got = y[..., 1::2].cpu().double()
    assert bool(((got / want - 1).abs()[number] <= 2.0 ** -11).all()) and bool(number.any(0).all())


@pytest.mark.parametrize("T,n", [(2000, 1), (2000, 3), (300, 1), (40, 3000)])
def test_recurrence_of_infinite_states_and_gradients(mem, T, n):
    """A state that is infinite stays so, with its sign, until an episode begins, and so does a gradient backwards, in one walk as in parts whose factors
    are below the smallest number; other channels are as without."""
    src = Source(T + 1, torch.float32)
    D, begin = 70, T * 3 // 4
    t = {k: src.normal(T, n, D) for k in ("x", "decay", "intake")}
    rate = torch.full((D,), -4.0, device="cuda")
    args, first = [plain(t[k]) for k in ("x", "decay", "intake")] + [rate], torch.zeros(T, n, dtype=torch.uint8, device="cuda")
    first[begin] = 1
    state, dstate = plain(src.normal(n, D)), plain(src.normal(n, D))
    want, want_h, saved = mem.gated_recurrence(*args, state=state, first=first, save=True)
    less = mem.gated_recurrence_backward(torch.ones_like(want), saved, *args, state=state, first=first, dstate=dstate)
    state[:, 3], state[:, 69], dstate[:, 5] = float("inf"), -float("inf"), float("inf")
    got, got_h, saved = mem.gated_recurrence(*args, state=state, first=first, save=True)
    assert bool((got[:begin, :, 3] == float("inf")).all()) and bool((got[:begin, :, 69] == -float("inf")).all())
    others = [c for c in range(D) if c not in (3, 69)]
    assert torch.equal(got[begin:], want[begin:]) and torch.equal(got_h, want_h) and torch.equal(got[..., others], want[..., others])
    g = mem.gated_recurrence_backward(torch.ones_like(want), saved, *args, state=state, first=first, dstate=dstate)
    assert bool((g.x[begin:, :, 5] == float("inf")).all()) and torch.equal(g.x[:begin], less.x[:begin])
    others = [c for c in range(D) if c != 5]
    assert torch.equal(g.x[..., others], less.x[..., others])
