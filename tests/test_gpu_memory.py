"""The policy memory operators against their definitions in 64 bits.

Tolerances.  An output of type X is rounded once: its unit roundoff times the value (2^-24 float32,
2^-8 bfloat16, 2^-11 float16, and half the smallest float16).  Before that it is a sum of m terms in
32 bits, every one of them right to some 16 roundings (products, an exponential whose argument is
at most a few units, a reciprocal), and the sum's own roundings grow as the square root of m; with
terms of either sign the sum of their sizes is about sqrt(m) times the largest sum.  So
32 * 2^-24 * sqrt(m) times the largest value of the tensor is allowed on top, m counted per output.
"""
import math

import pytest
import torch

import memory_reference as ref

pytestmark = pytest.mark.gpu

ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def mem():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2402_16801_amd import memory
    return memory


def close(what, got, want, terms):
    got64, want = got.detach().cpu().double(), want.detach()
    assert got64.shape == want.shape, (what, got64.shape, want.shape)
    assert bool(torch.isfinite(want).all()), what
    assert bool(torch.isfinite(got64).all()), f"{what} is not finite"
    big = float(want.abs().max()) if want.numel() else 0.0
    allowed = ROUND[got.dtype] * want.abs() + 32 * 2.0 ** -24 * math.sqrt(terms) * big + 2.0 ** -25
    over = (got64 - want).abs() - allowed
    assert bool((over <= 0).all()), f"{what}: off by {float((got64 - want).abs().max()):.3g} of {big:.3g}, worst {float(over.max()):.3g} over what is allowed"


def case_id(v):
    return "-".join(str(x) for x in v) if isinstance(v, tuple) else str(v)


class Source:
    """Random tensors on the CPU, in 64 bits but with values of the type they go to the GPU in."""

    def __init__(self, seed, dtype, order="time"):
        self.gen, self.dtype, self.order = torch.Generator().manual_seed(seed), dtype, order

    def normal(self, *shape, spread=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.gen) * spread).to(dtype).double()

    def seq(self, T, n, *width, spread=1.0):
        return self.normal(T, n, *width, spread=spread, dtype=self.dtype)

    def flags(self, T, n, p):
        return (torch.rand((T, n), generator=self.gen) < p).to(torch.uint8)

    def gpu(self, v, dtype=None):
        if v is None:
            return None
        if dtype is None:
            dtype = self.dtype
        if self.order == "batch" and v.dim() >= 3:
            return v.transpose(0, 1).contiguous().to("cuda", dtype).transpose(0, 1)
        if self.order == "slice" and v.dim() >= 3:       # inside a wider tensor, at an odd place
            wide = torch.full((v.shape[0], v.shape[1] + 1, v[0, 0].numel() + 7), float("nan"), dtype=dtype, device="cuda")
            part = wide[:, 1:, 3:3 + v[0, 0].numel()]
            part.copy_(v.reshape(v.shape[0], v.shape[1], -1))
            return part.unflatten(-1, v.shape[2:]) if v.dim() > 3 else part
        return v.to("cuda", dtype)


def plain(v):
    return None if v is None else v.to("cuda", torch.float32)


# ---- scan -----------------------------------------------------------------------------------------------

def scan_inputs(src, T, n, D, N, G, gate, carried):
    t = {"x": src.seq(T, n, D), "delta": src.seq(T, n, D, spread=0.7), "b": src.seq(T, n, G, N), "c": src.seq(T, n, G, N),
         "z": src.seq(T, n, D) if gate else None,
         "a": -torch.arange(1.0, N + 1, dtype=torch.float64).repeat(D, 1) * (1 + 0.05 * src.normal(D, N)), "d": src.normal(D),
         "delta_bias": -2.0 + src.normal(D), "state": src.normal(n, D, N) if carried else None}
    t["a"] = t["a"].float().double()
    t["delta_bias"] = t["delta_bias"].float().double()
    return t


def scan_gpu(src, t):
    g = {k: src.gpu(t[k]) for k in ("x", "delta", "b", "c", "z")}
    g.update({k: plain(t[k]) for k in ("a", "d", "delta_bias", "state")})
    return g


SCAN_CASES = [
    # dtype, T, n, D, N, G, order, gate, carried, begins, ragged
    ("f32", 1, 1, 1, 8, 1, "time", False, False, 0.0, False),
    ("f32", 1, 5, 70, 16, 1, "time", True, True, 0.5, False),
    ("bf16", 1, 3, 64, 32, 2, "slice", True, True, 0.5, False),
    ("f32", 2, 3, 65, 16, 1, "batch", True, False, 0.3, False),
    ("bf16", 7, 4, 64, 16, 1, "time", True, True, 0.3, False),
    ("f16", 8, 4, 128, 8, 2, "time", False, True, 0.1, False),
    ("f32", 9, 3, 130, 32, 2, "slice", True, True, 0.2, True),
    ("bf16", 17, 5, 96, 8, 4, "batch", True, False, 0.2, True),
    ("f16", 33, 2, 66, 32, 1, "time", True, True, 0.05, True),
    ("f32", 64, 2, 64, 16, 1, "time", False, True, 0.05, False),
    ("f32", 65, 2, 40, 16, 1, "batch", True, True, 0.05, True),
    ("bf16", 130, 3, 72, 16, 3, "slice", True, True, 0.03, True),
    ("f32", 300, 1, 64, 16, 1, "time", True, True, 0.0, False),
    ("f32", 300, 2, 70, 8, 1, "batch", True, False, 0.01, True),
    ("f16", 257, 1, 33, 32, 1, "slice", False, True, 0.02, False),
    ("f32", 24, 700, 64, 16, 1, "time", True, True, 0.02, True),     # several environments per wavefront of the backward pass
]


@pytest.mark.parametrize("case", SCAN_CASES, ids=case_id)
def test_scan_and_its_gradients(mem, case):
    dtype, T, n, D, N, G, order, gate, carried, begins, ragged = case
    src = Source(T * 1000 + D, TYPES[dtype], order)
    t = scan_inputs(src, T, n, D, N, G, gate, carried)
    first = src.flags(T, n, begins) if begins else None
    lengths = torch.tensor([(0, T, 1, T // 2)[i % 4] for i in range(n)], dtype=torch.int32) if ragged else None
    dy, dstate = src.seq(T, n, D), src.normal(n, D, N) if carried else None
    (y, h), want = ref.gradients(ref.scan, t, (dy, dstate), first=first, lengths=lengths)
    g = scan_gpu(src, t)
    how = {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    how["first"] = None if first is None else first.cuda()
    how["lengths"] = None if lengths is None else lengths.cuda()
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    got_y, got_h, nothing = mem.selective_scan(*args, **how)
    assert nothing is None
    chain = N * min(T, 64)
    close("y", got_y, y, chain)
    close("state", got_h, h, chain)
    again, last, saved = mem.selective_scan(*args, save=True, **how)
    close("y with saved states", again, y, chain)
    close("state with saved states", last, h, chain)
    got = mem.selective_scan_backward(src.gpu(dy), saved, *args, dstate=plain(dstate), **how)
    terms = {"b": chain + D // G, "c": chain + D // G, "a": chain + T * n, "d": T * n, "delta_bias": chain + T * n}
    for name, value in got._asdict().items():
        if value is None:
            assert t[name] is None, name
            continue
        close("gradient of " + name, value, want[name], terms.get(name, chain))


def test_scan_without_its_options(mem):
    """Step sizes as they are (no softplus, no bias, negative ones among them), no skip, no gate, no state."""
    src = Source(5, torch.float32)
    t = scan_inputs(src, 20, 3, 70, 16, 1, False, False)
    t["delta"] = t["delta"] * 0.1
    t["delta"] = t["delta"].float().double()
    t["d"] = t["delta_bias"] = None
    dy = src.seq(20, 3, 70)
    (y, h), want = ref.gradients(ref.scan, t, (dy, None), softplus=False)
    g = scan_gpu(src, t)
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    got_y, got_h, saved = mem.selective_scan(*args, softplus=False, save=True)
    close("y", got_y, y, 320)
    close("state", got_h, h, 320)
    got = mem.selective_scan_backward(src.gpu(dy), saved, *args, softplus=False)
    assert got.d is None and got.z is None and got.delta_bias is None and got.state is None
    for name in ("x", "delta", "a", "b", "c"):
        close("gradient of " + name, getattr(got, name), want[name], 400)


@pytest.mark.parametrize("T", [40, 200])
def test_scan_forgets_infinities_and_ignores_dead_steps(mem, T):
    """NaN and infinities in the carried state of an episode that is over, in the steps before the begin of another
    one, and behind the end of a sequence leave no trace elsewhere."""
    src = Source(11, torch.float32)
    n, D, N = 4, 70, 16
    t = scan_inputs(src, T, n, D, N, 1, True, True)
    first = torch.zeros(T, n, dtype=torch.uint8)
    first[0, 0] = first[17, 1] = first[0, 2] = first[1, 2] = first[T - 1, 3] = 1
    lengths = torch.tensor([T, T, T - 7, T], dtype=torch.int32)
    clean = {k: None if v is None else v.clone() for k, v in t.items()}
    t["state"][0], clean["state"][0] = float("inf"), 0.0
    t["state"][1], clean["state"][1] = float("nan"), 0.0
    for name in ("x", "b"):
        t[name][5, 1, ...], clean[name][5, 1, ...] = float("nan"), 0.0
    for name in ("x", "delta", "b", "c", "z"):
        t[name][T - 7:, 2], clean[name][T - 7:, 2] = float("nan"), 0.0
    dy = src.seq(T, n, D)
    bad_dy = dy.clone()
    bad_dy[T - 7:, 2] = float("nan")
    dy[:17, 1] = 0.0                        # what environment 1 answered before step 17 is not looked at
    bad_dy[:17, 1] = 0.0
    (y, h), want = ref.gradients(ref.scan, clean, (dy, None), first=first, lengths=lengths)
    g = scan_gpu(src, t)
    how = {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    how.update(first=first.cuda(), lengths=lengths.cuda())
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    got_y, got_h, saved = mem.selective_scan(*args, save=True, **how)
    seen = torch.ones(T, n, dtype=torch.bool)
    seen[:17, 1] = False
    close("y", got_y.cpu()[seen], y[seen], N * 64)
    close("state", got_h, h, N * 64)
    assert bool((got_y[T - 7:, 2] == 0).all())
    got = mem.selective_scan_backward(src.gpu(bad_dy), saved, *args, **how)
    for name in ("x", "delta", "b", "c", "z"):
        value = getattr(got, name).cpu()
        close("gradient of " + name, value[seen], want[name][seen], N * 64 + D)
        assert bool((value[T - 7:, 2] == 0).all())


@pytest.mark.parametrize("odd", ["b", "c", "both"])
@pytest.mark.parametrize("token", [True, False], ids=["token", "sequence"])
def test_scan_gradients_where_the_groups_are_the_outer_dimension(mem, token, odd):
    """b and c as views of [groups][..][states] tensors: the gradients are those of the same values laid out in order."""
    src = Source(45, torch.float32)
    T, n, D, N, G = (1 if token else 19), 5, 66, 16, 2
    t = scan_inputs(src, T, n, D, N, G, True, True)
    dy, dstate = src.seq(T, n, D), src.normal(n, D, N)
    _, want = ref.gradients(ref.scan, t, (dy, dstate))
    g = scan_gpu(src, t)
    for k in ("b", "c"):
        if odd in (k, "both"):
            g[k] = g[k].movedim(2, 0).contiguous().movedim(0, 2)
    dy = plain(dy)
    if token:
        g.update({k: g[k][0] for k in ("x", "delta", "b", "c", "z")})
        dy = dy[0]
    how = {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    _, _, saved = mem.selective_scan(*args, save=True, **how)
    got = mem.selective_scan_backward(dy, saved, *args, dstate=plain(dstate), **how)
    leaf = [v.requires_grad_(True) for v in args]
    y, h = mem.scan(*leaf, **how)
    auto = torch.autograd.grad([y, h], leaf, [dy, plain(dstate)])
    for name, value, same in zip(("x", "delta", "a", "b", "c"), got, auto):
        close("gradient of " + name, value[None] if token and name != "a" else value, want[name], N * min(T, 64) + D // G + T * n)
        assert torch.equal(value, same), name


@pytest.mark.parametrize("T", [5, 40, 300])
def test_scan_with_rates_of_minus_infinity(mem, T):
    """A state that nothing is left of after a step.  Steps behind the end, and places without a channel, leave it finite all the same."""
    src = Source(13, torch.float32)
    n, D, N = 3, 37, 16
    t = scan_inputs(src, T, n, D, N, 1, True, True)
    t["a"][-1, 3] = t["a"][5, :] = -float("inf")
    lengths = torch.tensor([T, T - 3, 1], dtype=torch.int32)
    dy, dstate = src.seq(T, n, D), src.normal(n, D, N)
    (y, h), want = ref.gradients(ref.scan, t, (dy, dstate), lengths=lengths)
    g = scan_gpu(src, t)
    how = {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    how["lengths"] = lengths.cuda()
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    got_y, got_h, saved = mem.selective_scan(*args, save=True, **how)
    close("y", got_y, y, N * 64)
    close("state", got_h, h, N * 64)
    got = mem.selective_scan_backward(plain(dy), saved, *args, dstate=plain(dstate), **how)
    for name in ("x", "b", "c", "d", "z", "state"):
        close("gradient of " + name, getattr(got, name), want[name], N * 64 + D + T * n)


def test_scan_steps_equal_the_sequence(mem):
    src = Source(21, torch.bfloat16)
    T, n, D, N, G = 40, 9, 136, 16, 2
    t = scan_inputs(src, T, n, D, N, G, True, True)
    first = src.flags(T, n, 0.1).cuda()
    g = scan_gpu(src, t)
    how = {k: g[k] for k in ("d", "z", "delta_bias")}
    whole, last, _ = mem.selective_scan(g["x"], g["delta"], g["a"], g["b"], g["c"], state=g["state"], first=first, **how)
    (want, h) = ref.scan(**{k: v for k, v in t.items()}, first=first.cpu())
    state = g["state"].clone()
    for s in range(T):
        y, same = mem.selective_scan_step(g["x"][s], g["delta"][s], g["a"], g["b"][s], g["c"][s], state, d=g["d"], z=g["z"][s],
                                          delta_bias=g["delta_bias"], first=first[s])
        assert same is state
        close(f"step {s}", y, want[s], N * 64)
    close("state", state, h, N * 64)
    close("state of the sequence", last, h, N * 64)
    # another place for the state, and two halves of the sequence
    out = torch.empty_like(state)
    before = state.clone()
    mem.selective_scan_step(g["x"][0], g["delta"][0], g["a"], g["b"][0], g["c"][0], state, out_state=out)
    assert torch.equal(before, state) and not torch.equal(out, state)
    _, mid, _ = mem.selective_scan(g["x"][:13], g["delta"][:13], g["a"], g["b"][:13], g["c"][:13], state=g["state"], first=first[:13], d=g["d"],
                                   z=g["z"][:13], delta_bias=g["delta_bias"])
    y, end, _ = mem.selective_scan(g["x"][13:], g["delta"][13:], g["a"], g["b"][13:], g["c"][13:], state=mid, first=first[13:], d=g["d"],
                                   z=g["z"][13:], delta_bias=g["delta_bias"])
    close("second half", y, want[13:], N * 64)
    close("its state", end, h, N * 64)


@pytest.mark.parametrize("dtype,n,D,N,G", [("bf16", 3001, 136, 16, 2), ("f32", 9001, 60, 8, 3), ("f16", 2003, 130, 32, 1)])
def test_scan_step_of_many_environments(mem, dtype, n, D, N, G):
    """A thread takes environments in turn, the next one's state under way while one is written in place."""
    src = Source(n + D, TYPES[dtype])
    t = scan_inputs(src, 1, n, D, N, G, True, True)
    g = scan_gpu(src, t)
    for flags in (src.flags(1, n, 0.3), None):
        y, h = ref.scan(**t, first=flags)
        held = g["state"].clone()
        got, same = mem.selective_scan_step(g["x"][0], g["delta"][0], g["a"], g["b"][0], g["c"][0], held, d=g["d"], z=g["z"][0], delta_bias=g["delta_bias"],
                                            first=None if flags is None else flags[0].cuda())
        assert same is held
        close("y", got, y[0], N * 64)
        close("state", held, h, N * 64)


@pytest.mark.parametrize("dtype,T,n,D,N,G", [("f32", 13, 2500, 130, 16, 2), ("bf16", 20, 3001, 40, 32, 1)])
def test_scan_of_many_environments(mem, dtype, T, n, D, N, G):
    """Blocks of the backward pass go on to further environments, of unequal lengths, with the gradients of a, d and delta_bias kept over them."""
    src = Source(n + D, TYPES[dtype])
    t = scan_inputs(src, T, n, D, N, G, True, True)
    first, lengths = src.flags(T, n, 0.1), torch.randint(0, T + 1, (n,), generator=src.gen, dtype=torch.int32)
    dy, dstate = src.seq(T, n, D), src.normal(n, D, N)
    (y, h), want = ref.gradients(ref.scan, t, (dy, dstate), first=first, lengths=lengths)
    g = scan_gpu(src, t)
    how = {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    how.update(first=first.cuda(), lengths=lengths.cuda())
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    got_y, got_h, saved = mem.selective_scan(*args, save=True, **how)
    close("y", got_y, y, N * T)
    close("state", got_h, h, N * T)
    got = mem.selective_scan_backward(src.gpu(dy), saved, *args, dstate=plain(dstate), **how)
    terms = {"b": N * T + D // G, "c": N * T + D // G, "a": N * T + T * n, "d": T * n, "delta_bias": N * T + T * n}
    for name, value in got._asdict().items():
        close("gradient of " + name, value, want[name], terms.get(name, N * T))


def test_scan_gradients_against_differences(mem):
    """Along a random direction of all inputs: central differences of step 2^-7 of the kernel's own forward pass.  Their
    error: the third derivative, some units times 2^-14 / 6, and the roundings of some 5,000 outputs of size 1
    (2^-24 each, of either sign) over 2^-7; together below 1 percent of slopes that are of the order of sqrt(5,000)."""
    src = Source(31, torch.float32)
    T, n, D, N = 18, 4, 70, 16
    t = scan_inputs(src, T, n, D, N, 1, True, True)
    first = src.flags(T, n, 0.05).cuda()
    w, wh = src.seq(T, n, D), src.normal(n, D, N)
    way = {k: 0.3 * src.normal(*v.shape) for k, v in t.items()}

    def loss(shift, save=False):
        g = {k: plain(v + shift * way[k]) for k, v in t.items()}
        args = [g.pop(k) for k in ("x", "delta", "a", "b", "c")]
        y, h, saved = mem.selective_scan(*args, first=first, save=save, **g)
        value = float((y.double().cpu() * w).sum() + (h.double().cpu() * wh).sum())
        return (value, args, g, saved) if save else value

    _, args, g, saved = loss(0.0, save=True)
    got = mem.selective_scan_backward(plain(w), saved, *args, first=first, dstate=plain(wh), **g)._asdict()
    slope = sum(float((got[k].double().cpu() * way[k]).sum()) for k in way)
    step = 2.0 ** -7
    difference = (loss(step) - loss(-step)) / (2 * step)
    size = math.sqrt(sum(float((got[k].double().cpu() * way[k]).pow(2).sum()) for k in way))
    assert abs(slope - difference) <= 0.01 * size, (slope, difference, size)


def test_scan_state_beyond_four_gigabytes(mem):
    """Offsets of the state pass 32 bits; the last environments come out as they do alone."""
    n, D, N = 70000, 1024, 16
    src = Source(41, torch.bfloat16)
    t = scan_inputs(src, 1, 3, D, N, 1, True, True)
    g = scan_gpu(src, t)
    state = torch.zeros(n, D, N, device="cuda")
    state[-3:] = g["state"]
    big = {k: torch.zeros((n,) + tuple(g[k].shape[2:]), dtype=torch.bfloat16, device="cuda") for k in ("x", "delta", "b", "c", "z")}
    for k in big:
        big[k][-3:] = g[k][0]
    y, state = mem.selective_scan_step(big["x"], big["delta"], g["a"], big["b"], big["c"], state, d=g["d"], z=big["z"], delta_bias=g["delta_bias"])
    small, small_state, _ = mem.selective_scan(g["x"], g["delta"], g["a"], g["b"], g["c"], d=g["d"], z=g["z"], delta_bias=g["delta_bias"], state=g["state"])
    assert torch.equal(y[-3:], small[0]) and torch.equal(state[-3:], small_state)
    assert bool((state[:-3] == 0).all()) and bool((y[:-3] == 0).all())


def test_scan_sums_of_groups_beyond_two_to_the_32_threads(mem):
    """64 steps of 4,096 environments of 512 groups of one channel: 2^32 sums for the gradients of b and c.  The environments are
    four, again and again, and come out as the four alone."""
    T, few, many, D, N = 64, 4, 4096, 512, 16
    src = Source(43, torch.bfloat16)
    t = scan_inputs(src, T, few, D, 16, 1, False, False)
    row = src.seq(T, 1, D, N)
    g = {k: src.gpu(t[k]) for k in ("x", "delta")}
    g.update({k: plain(t[k]) for k in ("a", "d", "delta_bias")})
    b, dy = src.gpu(row), src.gpu(src.seq(T, few, D))
    c = src.gpu(src.seq(T, 1, D, N))

    def gradients(n):
        x, delta, seed = (v.repeat(1, n // few, 1) for v in (g["x"], g["delta"], dy))
        args = (x, delta, g["a"], b.expand(T, n, D, N), c.expand(T, n, D, N))
        how = {"d": g["d"], "delta_bias": g["delta_bias"]}
        _, _, saved = mem.selective_scan(*args, save=True, **how)
        return mem.selective_scan_backward(seed, saved, *args, **how)

    small = gradients(few)
    big = gradients(many)
    for name in ("b", "c"):
        want, got = getattr(small, name), getattr(big, name)
        assert all(torch.equal(v, want) for v in got.split(few, 1)), name
    close("gradient of a", big.a, small.a.cpu().double() * (many // few), T * many)
    torch.cuda.empty_cache()


def test_scan_of_more_wavefronts_than_one_dimension_takes(mem):
    """2^26 + 2^16 groups of one channel, a wavefront each: forward and backward come out as 2^16 of them alone, again and again."""
    T, P, R, N = 2, 1 << 16, (1 << 10) + 1, 8
    src = Source(47, torch.bfloat16)
    t = scan_inputs(src, T, 1, P, N, 1, False, True)
    t["b"], t["c"] = src.seq(T, 1, P, N), src.seq(T, 1, P, N)
    g, dy = scan_gpu(src, t), src.gpu(src.seq(T, 1, P))

    def run(times):
        args = [g[k].repeat(1, 1, times, *[1] * (g[k].dim() - 3)) if k != "a" else g[k].repeat(times, 1) for k in ("x", "delta", "a", "b", "c")]
        how = {"state": g["state"].repeat(1, times, 1), "d": g["d"].repeat(times), "delta_bias": g["delta_bias"].repeat(times)}
        y, h, saved = mem.selective_scan(*args, save=True, **how)
        grads = mem.selective_scan_backward(dy.repeat(1, 1, times), saved, *args, **how)
        return {"y": y, "h": h, **{k: v for k, v in grads._asdict().items() if v is not None}}

    small = run(1)
    torch.cuda.empty_cache()
    for name, got in run(R).items():
        want = small[name]
        axis = {"y": 2, "h": 1, "x": 2, "delta": 2, "b": 2, "c": 2, "state": 1}.get(name, 0)
        assert all(torch.equal(v, want) for v in got.split(P, axis)), name
    del got
    torch.cuda.empty_cache()


def test_scan_of_groups_and_states_beyond_two_to_the_31(mem):
    """2^26 + 2^16 groups of one channel of 32 states: b and c of one step have more values than 31 bits count.  As 2^16 of them alone."""
    P, R, N = 1 << 16, (1 << 10) + 1, 32
    src = Source(53, torch.bfloat16)
    t = scan_inputs(src, 1, 1, P, N, 1, False, True)
    t["b"], t["c"] = src.seq(1, 1, P, N), src.seq(1, 1, P, N)
    g, dy = scan_gpu(src, t), src.gpu(src.seq(1, 1, P))

    def run(times):
        args = [g[k].repeat(1, 1, times, *[1] * (g[k].dim() - 3)) if k != "a" else g[k].repeat(times, 1) for k in ("x", "delta", "a", "b", "c")]
        how = {"d": g["d"].repeat(times), "delta_bias": g["delta_bias"].repeat(times)}
        state = g["state"].repeat(1, times, 1)
        out = {}
        out["y of a token"], out["state of a token"] = mem.selective_scan_step(args[0][0], args[1][0], args[2], args[3][0], args[4][0], state.clone(), **how)
        y, _, saved = mem.selective_scan(*args, state=state, save=True, **how)
        grads = mem.selective_scan_backward(dy.repeat(1, 1, times), saved, *args, state=state, **how)
        return {"y": y, **out, "x": grads.x, "delta": grads.delta, "b": grads.b, "c": grads.c, "a": grads.a, "state": grads.state}

    torch.cuda.empty_cache()
    small = run(1)
    for name, got in run(R).items():
        axis = {"y of a token": 1, "state of a token": 1, "a": 0, "state": 1}.get(name, 2)
        assert all(torch.equal(v, small[name]) for v in got.split(P, axis)), name
    del got
    torch.cuda.empty_cache()


# ---- convolution ------------------------------------------------------------------------------------------

CONV_CASES = [
    # dtype, T, n, D, K, order, carried, begins, ragged, silu, bias
    ("f32", 1, 1, 1, 2, "time", False, 0.0, False, True, True),
    ("bf16", 1, 5, 37, 4, "slice", True, 0.5, False, True, True),
    ("f16", 2, 3, 64, 4, "time", True, 0.4, False, True, False),
    ("f32", 3, 4, 7, 3, "batch", True, 0.3, True, False, True),
    ("bf16", 5, 6, 200, 4, "time", True, 0.3, True, True, True),
    ("f32", 8, 3, 33, 2, "slice", True, 0.2, True, True, True),
    ("f16", 9, 4, 65, 3, "batch", False, 0.2, False, True, True),
    ("bf16", 40, 3, 515, 4, "slice", True, 0.1, True, True, True),
    ("f32", 100, 2, 12, 4, "batch", True, 0.1, True, True, True),
    ("f16", 67, 1, 8, 2, "time", True, 0.0, False, False, False),
    ("f32", 12, 900, 24, 4, "time", True, 0.1, True, True, True),
]


@pytest.mark.parametrize("case", CONV_CASES, ids=case_id)
def test_conv_and_its_gradients(mem, case):
    dtype, T, n, D, K, order, carried, begins, ragged, silu, has_bias = case
    src = Source(T * 77 + D, TYPES[dtype], order)
    t = {"x": src.seq(T, n, D), "weight": src.normal(D, K, spread=0.5), "bias": src.normal(D) if has_bias else None,
         "state": src.normal(n, K - 1, D, dtype=TYPES[dtype]) if carried else None}
    first = src.flags(T, n, begins) if begins else None
    lengths = torch.tensor([(T, 0, 1, max(0, T - 2))[i % 4] for i in range(n)], dtype=torch.int32) if ragged else None
    dy, dstate = src.seq(T, n, D), src.normal(n, K - 1, D, dtype=TYPES[dtype])
    (y, tail), want = ref.gradients(ref.conv, t, (dy, dstate), first=first, lengths=lengths, silu=silu)
    how = {"state": None if t["state"] is None else t["state"].to("cuda", TYPES[dtype]), "silu": silu,
           "first": None if first is None else first.cuda(), "lengths": None if lengths is None else lengths.cuda()}
    args = (src.gpu(t["x"]), plain(t["weight"]), plain(t["bias"]))
    got_y, got_tail = mem.causal_conv(*args, **how)
    close("y", got_y, y, K + 1)
    assert torch.equal(got_tail.cpu().double(), tail)
    got = mem.causal_conv_backward(src.gpu(dy), *args, dstate=dstate.to("cuda", TYPES[dtype]), **how)
    for name, value in got._asdict().items():
        if value is None:
            assert t[name] is None, name
            continue
        close("gradient of " + name, value, want[name], T * n if name in ("weight", "bias") else 2 * K)
    # without a gradient of the new state, and bit for bit the same a second time
    _, want = ref.gradients(ref.conv, t, (dy, None), first=first, lengths=lengths, silu=silu)
    got = mem.causal_conv_backward(src.gpu(dy), *args, **how)
    close("gradient of x alone", got.x, want["x"], 2 * K)
    again = mem.causal_conv_backward(src.gpu(dy), *args, **how)
    assert torch.equal(got.x, again.x) and torch.equal(got.weight, again.weight)


def test_conv_steps_equal_the_sequence(mem):
    src = Source(3, torch.float16)
    T, n, D, K = 30, 7, 100, 4
    x, weight, bias, state = src.seq(T, n, D), src.normal(D, K), src.normal(D), src.normal(n, K - 1, D, dtype=torch.float16)
    first = src.flags(T, n, 0.15)
    want, tail = ref.conv(x, weight, bias, state, first)
    carried = state.to("cuda", torch.float16)
    for s in range(T):
        y, same = mem.causal_conv_step(src.gpu(x)[s], plain(weight), plain(bias), carried, first=first.cuda()[s])
        assert same is carried
        close(f"step {s}", y, want[s], K + 1)
    assert torch.equal(carried.cpu().double(), tail)


def test_conv_forgets_infinities_and_ignores_dead_steps(mem):
    src = Source(9, torch.float32)
    T, n, D, K = 30, 3, 20, 4
    x, weight, bias = src.seq(T, n, D), src.normal(D, K), src.normal(D)
    state = src.normal(n, K - 1, D)
    first, lengths = torch.zeros(T, n, dtype=torch.uint8), torch.tensor([T, T, 11], dtype=torch.int32)
    first[0, 0] = first[12, 1] = 1
    bad_x, bad_state = x.clone(), state.clone()
    bad_state[0], state[0] = float("nan"), 0.0
    bad_x[11, 1], x[11, 1] = float("inf"), 0.0
    bad_x[11:, 2] = float("nan")
    dy = src.seq(T, n, D)
    dy[11, 1] = 0.0
    (y, tail), want = ref.gradients(ref.conv, {"x": x, "weight": weight, "bias": bias, "state": state}, (dy, None), first=first, lengths=lengths, silu=False)
    how = {"state": plain(bad_state), "first": first.cuda(), "lengths": lengths.cuda(), "silu": False}
    got_y, got_tail = mem.causal_conv(plain(bad_x), plain(weight), plain(bias), **how)
    seen = torch.ones(T, n, dtype=torch.bool)
    seen[11, 1] = False
    close("y", got_y.cpu()[seen], y[seen], K + 1)
    assert bool((got_y[11:, 2] == 0).all()) and bool(torch.isfinite(got_tail).all())
    bad_dy = dy.clone()
    bad_dy[11:, 2] = float("nan")
    got = mem.causal_conv_backward(plain(bad_dy), plain(bad_x), plain(weight), plain(bias), **how)
    close("gradient of x", got.x, want["x"], 2 * K)
    close("gradient of the state", got.state, want["state"], 2 * K)
    close("gradient of bias", got.bias, want["bias"], T * n)


@pytest.mark.parametrize("dtype,T,n,D,K", [("bf16", 9, 5003, 260, 4), ("f32", 40, 2501, 67, 3), ("f16", 3, 30011, 30, 2)])
def test_conv_of_many_environments(mem, dtype, T, n, D, K):
    """Threads of the backward pass go on to further environments, with the gradients of weight and bias kept over them."""
    src = Source(n + D, TYPES[dtype])
    t = {"x": src.seq(T, n, D), "weight": src.normal(D, K, spread=0.5), "bias": src.normal(D), "state": src.normal(n, K - 1, D, dtype=TYPES[dtype])}
    first, lengths = src.flags(T, n, 0.15), torch.randint(0, T + 1, (n,), generator=src.gen, dtype=torch.int32)
    dy, dstate = src.seq(T, n, D), src.normal(n, K - 1, D, dtype=TYPES[dtype])
    for flags in (first, None):
        (y, tail), want = ref.gradients(ref.conv, t, (dy, dstate), first=flags, lengths=lengths)
        how = {"state": t["state"].to("cuda", TYPES[dtype]), "first": None if flags is None else flags.cuda(), "lengths": lengths.cuda()}
        args = (src.gpu(t["x"]), plain(t["weight"]), plain(t["bias"]))
        got_y, got_tail = mem.causal_conv(*args, **how)
        close("y", got_y, y, K + 1)
        assert torch.equal(got_tail.cpu().double(), tail)
        got = mem.causal_conv_backward(src.gpu(dy), *args, dstate=dstate.to("cuda", TYPES[dtype]), **how)
        for name, value in got._asdict().items():
            close("gradient of " + name, value, want[name], T * n if name in ("weight", "bias") else 2 * K)


@pytest.mark.parametrize("dtype,n,D,K", [("bf16", 2000, 1027, 4), ("f32", 5001, 516, 3), ("f16", 60001, 13, 2)])
def test_conv_step_of_many_environments(mem, dtype, n, D, K):
    """A thread takes environments in turn, the next one's state under way while one is written in place."""
    src = Source(n + D, TYPES[dtype])
    x, weight, bias, state = src.seq(1, n, D), src.normal(D, K, spread=0.5), src.normal(D), src.normal(n, K - 1, D, dtype=TYPES[dtype])
    for flags in (src.flags(1, n, 0.3), None):
        y, tail = ref.conv(x, weight, bias, state, flags)
        held = state.to("cuda", TYPES[dtype])
        got, same = mem.causal_conv_step(src.gpu(x)[0], plain(weight), plain(bias), held, first=None if flags is None else flags[0].cuda())
        assert same is held
        close("y", got, y[0], K + 1)
        assert torch.equal(held.cpu().double(), tail)


def test_conv_gradients_against_differences(mem):
    """As for the scan: central differences of step 2^-7 along a random direction, good to 1 percent."""
    src = Source(13, torch.float32)
    T, n, D, K = 25, 4, 60, 4
    t = {"x": src.seq(T, n, D), "weight": src.normal(D, K), "bias": src.normal(D), "state": src.normal(n, K - 1, D)}
    first = src.flags(T, n, 0.1).cuda()
    w, wt = src.seq(T, n, D), src.normal(n, K - 1, D)
    way = {k: 0.3 * src.normal(*v.shape) for k, v in t.items()}

    def loss(shift):
        g = {k: plain(v + shift * way[k]) for k, v in t.items()}
        y, tail = mem.causal_conv(g["x"], g["weight"], g["bias"], state=g["state"], first=first)
        return float((y.double().cpu() * w).sum() + (tail.double().cpu() * wt).sum())

    g = {k: plain(v) for k, v in t.items()}
    got = mem.causal_conv_backward(plain(w), g["x"], g["weight"], g["bias"], state=g["state"], first=first, dstate=plain(wt))._asdict()
    slope = sum(float((got[k].double().cpu() * way[k]).sum()) for k in way)
    size = math.sqrt(sum(float((got[k].double().cpu() * way[k]).pow(2).sum()) for k in way))
    difference = (loss(2.0 ** -7) - loss(-2.0 ** -7)) * 2.0 ** 6
    assert abs(slope - difference) <= 0.01 * size, (slope, difference, size)


def test_conv_beyond_two_to_the_31_elements(mem):
    T, n, D, K = 33, 65536, 1000, 4
    x = torch.zeros(T, n, D, dtype=torch.bfloat16, device="cuda")
    src = Source(17, torch.bfloat16)
    part = src.gpu(src.seq(T, 2, D))
    weight = plain(src.normal(D, K))
    x[:, -2:] = part
    y, tail = mem.causal_conv(x, weight)
    small, small_tail = mem.causal_conv(part.contiguous(), weight)
    assert torch.equal(y[:, -2:], small) and torch.equal(tail[-2:], small_tail)
    assert int((y[:, :-2] != 0).sum(dtype=torch.int64)) == 0


def test_conv_step_of_the_most_environments(mem):
    """2^31 - 4096 environments of one channel, a state in place: 4,096 of them, again and again."""
    few, times = 4096, 2 ** 19 - 1
    src = Source(23, torch.bfloat16)
    x, state, weight = (src.normal(few, 1, dtype=torch.bfloat16).cuda().bfloat16(), src.normal(few, 1, 1, dtype=torch.bfloat16).cuda().bfloat16(),
                        plain(src.normal(1, 2)))
    want, after = mem.causal_conv_step(x, weight, None, state, out_state=torch.empty_like(state))
    held = state.repeat(times, 1, 1)
    y, same = mem.causal_conv_step(x.repeat(times, 1), weight, None, held)
    assert same is held
    for got, one in ((y, want), (held, after)):
        assert all(torch.equal(v, one.view(1, few).expand_as(v)) for v in got.view(times, few).split(1 << 14))
    del y, held, same, got
    torch.cuda.empty_cache()


# ---- norm -------------------------------------------------------------------------------------------------

NORM_CASES = [
    # dtype, residual, T, n, D, order, gate, act, post, scale, pre, dout
    ("f32", "f32", 1, 1, 1, "time", True, "sigmoid", True, True, True, True),
    ("f32", "f32", 1, 3, 3, "time", False, "sigmoid", True, False, True, True),
    ("bf16", "bf16", 2, 5, 7, "slice", True, "silu", True, True, True, True),
    ("bf16", "f32", 3, 4, 512, "time", True, "sigmoid", True, True, True, True),
    ("f16", "f16", 3, 5, 200, "batch", True, "linear", True, True, False, False),
    ("f32", "f32", 2, 7, 1345, "time", True, "sigmoid", True, True, True, True),
    ("f16", "f32", 2, 3, 1025, "slice", True, "sigmoid", False, True, True, True),
    ("bf16", "bf16", 5, 9, 1000, "time", False, "sigmoid", False, False, True, True),
    ("f32", "f32", 3, 3, 2050, "slice", True, "silu", True, True, True, True),
    ("bf16", "bf16", 2, 3, 4097, "batch", True, "sigmoid", True, True, True, True),
    ("f32", "f32", 1, 3, 8192, "time", True, "sigmoid", True, True, True, True),
    ("f16", "f16", 1, 2, 8191, "time", True, "sigmoid", True, True, True, True),
    ("f32", "f32", 50, 300, 20, "time", True, "sigmoid", True, True, True, True),
]


@pytest.mark.parametrize("case", NORM_CASES, ids=case_id)
def test_norm_and_its_gradients(mem, case):
    dtype, residual_dtype, T, n, D, order, gate, act, post, scale, pre, has_dout = case
    src, rtype = Source(T * 31 + D, TYPES[dtype], order), TYPES[residual_dtype]
    t = {"y": src.seq(T, n, D), "residual": src.normal(T, n, D, spread=2.0, dtype=rtype), "gate": src.seq(T, n, D) if gate else None,
         "post_weight": 1 + src.normal(D, spread=0.1) if post else None, "scale": src.normal(D) if scale else None,
         "pre_weight": 1 + src.normal(D, spread=0.1) if pre else None}
    t = {k: v if v is None or k in ("y", "residual", "gate") else v.float().double() for k, v in t.items()}
    dout, du = src.normal(T, n, D, dtype=rtype) if has_dout else None, src.seq(T, n, D)
    (out, u), want = ref.gradients(ref.norm, t, (dout, du), gate_act=act, eps=1e-5)
    g = {"y": src.gpu(t["y"]), "residual": src.gpu(t["residual"], rtype), "gate": src.gpu(t["gate"]),
         **{k: plain(t[k]) for k in ("post_weight", "scale", "pre_weight")}}
    how = {k: g[k] for k in ("gate", "post_weight", "scale", "pre_weight")}
    got_out, got_u = mem.residual_norm(g["y"], g["residual"], gate_act=act, eps=1e-5, **how)
    assert got_out.dtype == rtype
    close("out", got_out, out, 4)
    close("u", got_u, u, 4)
    got = mem.residual_norm_backward(src.gpu(dout, rtype), src.gpu(du), g["y"], g["residual"], gate_act=act, eps=1e-5, **how)
    for name, value in got._asdict().items():
        if value is None:
            assert t[name] is None, name
            continue
        close("gradient of " + name, value, want[name], T * n if name in ("post_weight", "scale", "pre_weight") else 16)


def test_norm_of_rows_of_zeros_and_of_two_dimensions(mem):
    """A row of zeros has the root 1 / sqrt(eps); [rows][channels] is taken as one step."""
    src = Source(2, torch.float32)
    y, r = src.normal(6, 130), src.normal(6, 130)
    y[2] = r[2] = 0.0
    y[4] = 0.0
    w = src.normal(130)
    out, u = ref.norm(y, r, post_weight=w, pre_weight=w)
    got_out, got_u = mem.residual_norm(plain(y), plain(r), post_weight=plain(w), pre_weight=plain(w))
    close("out", got_out, out, 4)
    close("u", got_u, u, 4)
    assert bool((got_u[2] == 0).all())
    du = src.normal(6, 130, spread=1e-3)
    _, want = ref.gradients(ref.norm, {"y": y, "residual": r, "post_weight": w, "pre_weight": w}, (None, du))
    got = mem.residual_norm_backward(None, plain(du), plain(y), plain(r), post_weight=plain(w), pre_weight=plain(w))
    for name in ("y", "residual", "post_weight", "pre_weight"):
        close("gradient of " + name, getattr(got, name), want[name], 16)


@pytest.mark.parametrize("D", [1, 200, 512, 1345])
@pytest.mark.parametrize("power", [-149, -132, -126])
def test_norm_with_a_subnormal_eps(mem, D, power):
    """Rows of zeros, rows whose squares are subnormal (and exact in 32 bits), and ordinary ones."""
    src = Source(D - power, torch.float32)
    y, r, w = src.normal(3, D), src.normal(3, D), (1 + src.normal(D, spread=0.1)).float().double()
    y[0] = r[0] = r[1] = 0.0
    y[1] = 2.0 ** -66
    how = {"post_weight": w, "pre_weight": w}
    out, u = ref.norm(y, r, eps=2.0 ** power, **how)
    got_out, got_u = mem.residual_norm(plain(y), plain(r), eps=2.0 ** power, **{k: plain(v) for k, v in how.items()})
    close("out", got_out, out, 4)
    close("u", got_u, u, 4)
    assert bool((got_out[0] == 0).all()) and bool((got_u[0] == 0).all())
    y, r, du = y[2:], r[2:], src.normal(1, D)
    _, want = ref.gradients(ref.norm, {"y": y, "residual": r, **how}, (None, du), eps=2.0 ** power)
    got = mem.residual_norm_backward(None, plain(du), plain(y), plain(r), eps=2.0 ** power, **{k: plain(v) for k, v in how.items()})
    for name in ("y", "residual", "post_weight", "pre_weight"):
        close("gradient of " + name, getattr(got, name), want[name], 16)


def alike(what, got, want, terms):
    """close(), where the definition is finite; where it is infinite or no number, the same."""
    got64 = got.detach().cpu().double()
    assert torch.equal(torch.isnan(got64), torch.isnan(want)), f"{what}: {int(torch.isnan(got64).sum())} values are no numbers, by its definition {int(torch.isnan(want).sum())}"
    ends = torch.isinf(want)
    assert torch.equal(torch.isinf(got64), ends) and torch.equal(got64[ends], want[ends]), f"{what}: infinities differ"
    finite = torch.isfinite(want)
    close(what, torch.where(finite, got.detach().cpu(), 0.0), torch.where(finite, want, 0.0), terms)


# lengths that fill the lanes of a row (512), that do not in one of one, two and four chunks a lane, that leave lanes without a value, and short ones
@pytest.mark.parametrize("D", [3, 7, 20, 200, 300, 512, 513, 600, 1000, 1345, 1544, 2050, 3000, 4097, 6000, 8191])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_rows_with_an_infinity(mem, dtype, D):
    """An infinity makes the root of its row 0: the row's other values are the residual's, or 0, wherever it lies.  One in the
    gradient of u is in that of every value of its row and of no other row."""
    src = Source(D, TYPES[dtype])
    places = sorted({0, 1, D // 2, max(0, D - 9), D - 2, D - 1})
    n = len(places) + 1                                   # the last row is finite
    t = {"y": src.seq(1, n, D), "residual": src.seq(1, n, D), "gate": src.seq(1, n, D), "pre_weight": 1 + src.normal(D, spread=0.1),
         "post_weight": 1 + src.normal(D, spread=0.1)}
    t = {k: v.float().double() for k, v in t.items()}
    du = src.seq(1, n, D)

    def put(v):
        v = v.clone()
        for row, place in enumerate(places):
            v[0, row, place] = float("inf") if row % 2 else -float("inf")
        return v

    for where, post in (("y", True), ("y", False), ("residual", True)):
        bad = {k: put(v) if k == where else v for k, v in t.items() if post or k != "post_weight"}
        out, u = ref.norm(**bad)
        got_out, got_u = mem.residual_norm(**{k: plain(v) if "weight" in k else src.gpu(v) for k, v in bad.items()})
        alike(f"out, infinity in {where}", got_out, out, 4)
        alike(f"u, infinity in {where}", got_u, u, 4)
    t.pop("post_weight")
    _, want = ref.gradients(ref.norm, t, (None, put(du)))
    got = mem.residual_norm_backward(None, src.gpu(put(du)), src.gpu(t["y"]), src.gpu(t["residual"]), gate=src.gpu(t["gate"]), pre_weight=plain(t["pre_weight"]))
    for name in ("y", "residual", "gate"):
        alike("gradient of " + name, getattr(got, name), want[name], 16)


@pytest.mark.parametrize("rows", [1, 2, 3, 5])
@pytest.mark.parametrize("D", [6, 512, 700, 1345])
def test_norm_gradients_of_weights_with_an_infinity_in_the_last_row(mem, D, rows):
    """Rows that a block has no place filled with add nothing: an infinite gradient in the last row is in the weights' gradients once."""
    src = Source(100 * D + rows, torch.float32)
    t = {"y": src.seq(1, rows, D), "residual": src.seq(1, rows, D), "scale": src.normal(D), "pre_weight": (1 + src.normal(D, spread=0.1)).float().double()}
    du = src.seq(1, rows, D)
    du[0, -1, D // 2] = float("inf")
    _, want = ref.gradients(ref.norm, t, (None, du))
    got = mem.residual_norm_backward(None, plain(du), plain(t["y"]), plain(t["residual"]), scale=plain(t["scale"]), pre_weight=plain(t["pre_weight"]))
    for name in ("scale", "pre_weight"):
        alike("gradient of " + name, getattr(got, name), want[name], rows + 16)


def _norm_tensors(src, T, n, D, gate=True):
    t = {"y": src.seq(T, n, D), "residual": src.seq(T, n, D), "gate": src.seq(T, n, D) if gate else None, "scale": src.normal(D),
         "post_weight": (1 + src.normal(D, spread=0.1)).float().double(), "pre_weight": (1 + src.normal(D, spread=0.1)).float().double()}
    return {k: v for k, v in t.items() if v is not None}


# rows of one, two, four and eight wavefronts, forward and backward, whole, in vectors and ragged; more of them than the chip holds at
# once, and no multiple of that
@pytest.mark.parametrize("dtype,rows,D", [("f32", 27001, 9), ("bf16", 26003, 512), ("f32", 13001, 333), ("bf16", 9007, 1000), ("f32", 7001, 1345), ("f16", 5003, 1536),
                                          ("bf16", 3301, 2050), ("f32", 2003, 3000), ("bf16", 1999, 4097), ("f32", 1801, 6000)])
def test_norm_of_many_rows(mem, dtype, rows, D):
    """Blocks go on to further rows: what they read ahead, and the sums in LDS that several wavefronts share, row after row."""
    src = Source(rows + D, TYPES[dtype])
    t = _norm_tensors(src, 1, rows, D)
    dout, du = src.seq(1, rows, D), src.seq(1, rows, D)
    (out, u), want = ref.gradients(ref.norm, t, (dout, du))
    g = {k: plain(v) if k in ("scale", "post_weight", "pre_weight") else src.gpu(v) for k, v in t.items()}
    got_out, got_u = mem.residual_norm(**g)
    close("out", got_out, out, 4)
    close("u", got_u, u, 4)
    got = mem.residual_norm_backward(src.gpu(dout), src.gpu(du), **g)
    for name, value in got._asdict().items():
        close("gradient of " + name, value, want[name], rows if name in ("post_weight", "scale", "pre_weight") else 16)


def test_norm_gradients_against_differences(mem):
    """As for the scan: central differences of step 2^-7 along a random direction, good to 1 percent."""
    src = Source(19, torch.float32)
    T, n, D = 6, 5, 130
    t = {"y": src.seq(T, n, D), "residual": src.seq(T, n, D), "gate": src.seq(T, n, D), "post_weight": 1 + src.normal(D, spread=0.1),
         "scale": src.normal(D), "pre_weight": 1 + src.normal(D, spread=0.1)}
    w, wu = src.seq(T, n, D), src.seq(T, n, D)
    way = {k: 0.3 * src.normal(*v.shape) for k, v in t.items()}

    def loss(shift):
        out, u = mem.residual_norm(**{k: plain(v + shift * way[k]) for k, v in t.items()})
        return float((out.double().cpu() * w).sum() + (u.double().cpu() * wu).sum())

    got = mem.residual_norm_backward(plain(w), plain(wu), **{k: plain(v) for k, v in t.items()})._asdict()
    slope = sum(float((got[k].double().cpu() * way[k]).sum()) for k in way)
    size = math.sqrt(sum(float((got[k].double().cpu() * way[k]).pow(2).sum()) for k in way))
    difference = (loss(2.0 ** -7) - loss(-2.0 ** -7)) * 2.0 ** 6
    assert abs(slope - difference) <= 0.01 * size, (slope, difference, size)


# ---- streams, graphs, autograd -----------------------------------------------------------------------------

def _all_operators(mem, g, first, work):
    y, tail = mem.causal_conv(g["x"], work["weight"], None, first=first)
    y, h, saved = mem.selective_scan(y, g["delta"], g["a"], g["b"], g["c"], d=g["d"], z=g["z"], delta_bias=g["delta_bias"], state=g["state"],
                                     first=first, save=True)
    out, u = mem.residual_norm(y, g["x"], gate=g["z"], post_weight=g["d"])
    dn = mem.residual_norm_backward(out, u, y, g["x"], gate=g["z"], post_weight=g["d"])
    ds = mem.selective_scan_backward(dn.y, saved, y, g["delta"], g["a"], g["b"], g["c"], d=g["d"], z=g["z"], delta_bias=g["delta_bias"],
                                     state=g["state"], first=first)
    dc = mem.causal_conv_backward(ds.x, g["x"], work["weight"], None, first=first)
    return [v for v in (y, tail, h, out, u, *dn, *ds, *dc) if v is not None]


def test_operators_on_another_stream_and_in_a_graph(mem):
    """On a side stream, and captured once and replayed with other inputs in the same tensors: bit for bit as eager."""
    src = Source(51, torch.bfloat16)
    T, n, D, N = 150, 2, 96, 16
    sets = [scan_gpu(src, scan_inputs(src, T, n, D, N, 1, True, True)) for _ in range(3)]
    first = src.flags(T, n, 0.05).cuda()
    work = {"weight": plain(src.normal(D, 4))}
    want = [[v.clone() for v in _all_operators(mem, s, first, work)] for s in sets]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _all_operators(mem, sets[0], first, work)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    held = {k: v.clone() for k, v in sets[0].items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all_operators(mem, held, first, work)
    for k in (1, 2, 0, 1):
        for name in held:
            held[name].copy_(sets[k][name])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[k])), k
        mem.causal_conv(sets[0]["x"], work["weight"])
        torch.cuda.synchronize()


def test_operators_give_the_same_bits_every_time(mem):
    src = Source(61, torch.float32)
    g = scan_gpu(src, scan_inputs(src, 70, 40, 130, 16, 2, True, True))
    first = src.flags(70, 40, 0.05).cuda()
    work = {"weight": plain(src.normal(130, 3))}
    runs = [_all_operators(mem, g, first, work) for _ in range(3)]
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_differentiable_functions(mem):
    """conv, scan and norm chained under autograd against the same chain in 64 bits.  The values that go from one to the next
    are float32, so the tolerance is that of three sums in a row."""
    src = Source(71, torch.float32)
    T, n, D, N = 12, 3, 66, 16
    t = scan_inputs(src, T, n, D, N, 1, True, True)
    t["weight"], t["post"], t["tail"] = src.normal(D, 4), src.normal(D), src.normal(n, 3, D)
    first = src.flags(T, n, 0.1)
    w = src.seq(T, n, D)

    def chain(f, p, flags):
        x, tail = f.conv(p["x"], p["weight"], state=p["tail"], first=flags)
        y, h = f.scan(x, p["delta"], p["a"], p["b"], p["c"], d=p["d"], z=p["z"], delta_bias=p["delta_bias"], state=p["state"], first=flags)
        out, u = f.norm(y, p["x"], gate=p["z"], post_weight=p["post"])
        return out, u, h, tail

    def grads(f, p, flags, weight):
        p = {k: v.detach().clone().requires_grad_(True) for k, v in p.items()}
        out, u, h, tail = chain(f, p, flags)
        ((out + 2 * u) * weight).sum().add(h.sum()).add(tail.sum()).backward()
        return {k: v.grad for k, v in p.items()}

    want = grads(ref, t, first, w)
    got = grads(mem, {k: plain(v) for k, v in t.items()}, first.cuda(), plain(w))
    for name in want:
        close("gradient of " + name, got[name], want[name], 9 * (N * T + T * n + D))


@pytest.mark.parametrize("grad", [True, False], ids=["grad", "no_grad"])
def test_scan_keeps_nothing_where_no_backward_pass_can_follow(mem, grad):
    """Under no_grad, and where nothing requires gradients, no states are saved: 16 floats for every 8 steps, twice the outputs."""
    src = Source(95, torch.float32)
    T, n, D = 256, 16, 512
    g = scan_gpu(src, scan_inputs(src, T, n, D, 16, 1, True, True))
    args, how = [g[k] for k in ("x", "delta", "a", "b", "c")], {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    want_y, want_h = mem.scan(*[v.clone().requires_grad_(True) for v in args], **how)
    assert want_y.requires_grad and want_h.requires_grad
    want_y, want_h = want_y.detach(), want_h.detach()
    if not grad:
        args[0].requires_grad_(True)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    with torch.set_grad_enabled(grad):
        y, h = mem.scan(*args, **how)
    saved = T // 8 * n * D * 16 * 4
    taken = torch.cuda.max_memory_allocated() - held
    assert taken < saved / 2 + y.numel() * 4 + h.numel() * 4, (taken, saved)
    assert not y.requires_grad and torch.equal(y, want_y) and torch.equal(h, want_h)


def _rollout_and_step(mem, operator):
    """(a rollout from a state as a differentiable call, a step that takes a state and out_state, a fresh state, its leaves)"""
    src = Source(91, torch.float32)
    T, n, D, N = 6, 3, 40, 16
    t = scan_inputs(src, T, n, D, N, 1, False, True)
    g = scan_gpu(src, t)
    if operator == "conv":
        weight = plain(src.normal(D, 4)).requires_grad_(True)
        return (lambda s: mem.conv(g["x"], weight, state=s)[0], lambda s, out=None: mem.causal_conv_step(g["x"][0], weight, None, s, out_state=out)[1],
                plain(src.normal(n, 3, D)), weight)
    x = g["x"].requires_grad_(True)
    return (lambda s: mem.scan(x, g["delta"], g["a"], g["b"], g["c"], state=s)[0],
            lambda s, out=None: mem.selective_scan_step(g["x"][0], g["delta"][0], g["a"], g["b"][0], g["c"][0], s, out_state=out)[1], g["state"], x)


@pytest.mark.parametrize("operator", ["conv", "scan"])
def test_a_step_between_forward_and_backward(mem, operator):
    """A state that a rollout began with is stepped on before the backward pass.  The convolution's gradients need it as it was, so
    that they raise as behind PyTorch's own operations in place; the scan's do not, and are what they are without the step."""
    rollout, step, state, leaf = _rollout_and_step(mem, operator)
    (want,) = torch.autograd.grad(rollout(state).sum(), leaf)
    y = rollout(state)
    step(state.clone())
    step(state, torch.empty_like(state))
    (same,) = torch.autograd.grad(y.sum(), leaf, retain_graph=True)
    assert torch.equal(same, want)
    before = state.clone()
    assert step(state) is state and not torch.equal(state, before)
    if operator == "conv":
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    else:
        (same,) = torch.autograd.grad(y.sum(), leaf)
        assert torch.equal(same, want)
    # written as another state's place, too
    y, other = rollout(state), state.clone()
    step(other, state)
    if operator == "conv":
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


@pytest.mark.parametrize("operator", ["conv", "scan"])
def test_states_written_in_place_as_autograd_sees_them(mem, operator):
    from paper_2402_16801_amd import binding
    _, step, state, _ = _rollout_and_step(mem, operator)
    version = state._version
    step(state)
    assert state._version == version + 1
    step(state, torch.empty_like(state))
    with pytest.raises(binding.CraftaxError):
        step(state[:, :-1])
    assert state._version == version + 1
    for grown in (state.clone().requires_grad_(True), state.clone().requires_grad_(True) * 2):
        kept = grown.detach().clone()
        for where in ((grown,), (state, grown)):
            with pytest.raises(binding.CraftaxError, match="requires gradients"):
                step(*where)
        torch.cuda.synchronize()
        assert torch.equal(grown, kept) and step(grown, torch.empty_like(state)) is not grown
        with torch.no_grad():
            assert step(grown) is grown and not torch.equal(grown, kept)
    with torch.inference_mode():
        plain_state = state.clone()
        assert step(plain_state) is plain_state
    assert step(plain_state) is plain_state


# ---- refusals ---------------------------------------------------------------------------------------------

def test_refusals(mem):
    from paper_2402_16801_amd import binding
    src = Source(81, torch.float32)
    g = scan_gpu(src, scan_inputs(src, 4, 3, 32, 16, 2, True, True))
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    w = plain(src.normal(32, 4))

    def refused(text, call, *a, **k):
        with pytest.raises(binding.CraftaxError, match=text):
            call(*a, **k)

    refused("no CPU path", mem.causal_conv, g["x"].cpu(), w)
    refused("float32, bfloat16 or float16", mem.causal_conv, g["x"].double(), w)
    refused("taps must be 2..4", mem.causal_conv, g["x"], plain(src.normal(32, 5)))
    refused("weight", mem.causal_conv, g["x"], w[:31])
    refused("side by side", mem.causal_conv, g["x"].transpose(1, 2).contiguous().transpose(1, 2), w)
    refused("first must be", mem.causal_conv, g["x"], w, first=torch.zeros(4, 3, device="cuda"))
    refused("first has shape", mem.causal_conv, g["x"], w, first=torch.zeros(3, 4, dtype=torch.uint8, device="cuda"))
    refused("lengths", mem.causal_conv, g["x"], w, lengths=torch.zeros(3, dtype=torch.int64, device="cuda"))
    refused("state", mem.causal_conv, g["x"], w, state=torch.zeros(3, 2, 32, device="cuda"))
    refused("steps, n and channels must be positive", mem.causal_conv, g["x"][:0], w)
    refused("delta has shape", mem.selective_scan, args[0], args[1][:3], *args[2:])
    refused("delta is", mem.selective_scan, args[0], args[1].half(), *args[2:])
    refused("c has shape", mem.selective_scan, *args[:4], args[4][..., :8])
    refused("states must be 8, 16 or 32", mem.selective_scan, args[0], args[1], args[2][:, :4].contiguous(), args[3][..., :4], args[4][..., :4])
    refused("groups must divide", mem.selective_scan, args[0], args[1], args[2], torch.zeros(4, 3, 3, 16, device="cuda"), torch.zeros(4, 3, 3, 16, device="cuda"))
    refused("saved is not", mem.selective_scan_backward, g["x"], None, *args)
    refused("saved is not", mem.selective_scan_backward, g["x"], torch.zeros(8, dtype=torch.uint8, device="cuda"), *args)
    odd = torch.zeros(32 * 16 + 1, device="cuda")[1:].view(32, 16)
    refused("16-byte aligned", mem.selective_scan, args[0], args[1], odd, *args[3:])
    refused("residual must be", mem.residual_norm, g["x"], g["x"].half())
    refused("gate_act", mem.residual_norm, g["x"], g["x"], gate_act="relu")
    refused("eps must be positive", mem.residual_norm, g["x"], g["x"], eps=0.0)
    wide = torch.zeros(1, 1, 8193, device="cuda")
    refused("channels must be 1..8192", mem.residual_norm, wide, wide)


def test_options_without_a_truth_value_are_refused(mem):
    src = Source(83, torch.float32)
    g, w = scan_gpu(src, scan_inputs(src, 4, 3, 32, 16, 2, True, True)), plain(src.normal(32, 4))
    args, neither = [g[k] for k in ("x", "delta", "a", "b", "c")], torch.zeros(2)
    for call in (lambda: mem.causal_conv(g["x"], w, silu=neither), lambda: mem.selective_scan(*args, softplus=neither),
                 lambda: mem.selective_scan(*args, save=neither)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()


def test_counts_that_32_bits_do_not_hold_are_refused(mem):
    """2^32 + 3 taps are not three, nor 2^32 + 16 states sixteen."""
    from paper_2402_16801_amd import binding
    x, wide = torch.zeros(1, 1, 1, device="cuda"), torch.empty(1, 2 ** 32 + 16, device="cuda")
    with pytest.raises(binding.CraftaxError, match="taps is beyond"):
        mem.causal_conv(x, wide[:, :2 ** 32 + 3])
    short = wide.view(1, 1, 1, -1)
    with pytest.raises(binding.CraftaxError, match="states is beyond"):
        mem.selective_scan(x, x, wide, short, short)
    del wide, short
    torch.cuda.empty_cache()


def test_want_of_memory_is_the_error_that_torch_has_for_it(mem):
    """Outputs of 550 GB, of an input that is one row: what a caller who tries again with less looks for."""
    x, weight = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda").expand(1 << 26, 64, 64), torch.zeros(64, 4, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        mem.causal_conv(x, weight)
    y, _ = mem.causal_conv(x[:4], weight)
    assert bool((y == 0).all())


def test_refusals_at_the_c_entry(mem):
    """Codes and texts of the calls themselves; nothing is launched."""
    import ctypes
    from paper_2402_16801_amd import binding as cx
    lib = cx.load()
    for name in ("causal_conv", "causal_conv_backward", "selective_scan", "selective_scan_backward", "residual_norm", "residual_norm_backward"):
        assert getattr(lib, "craftax_" + name)(None, None) == -1
    v = torch.zeros(64, device="cuda")
    p = v.data_ptr()
    conv = cx.ConvArgs(dtype=0, steps=1, n=1, channels=4, taps=4, weight=p, x=p, y=p)
    assert lib.craftax_causal_conv(conv, None) == 0
    for field, value, code in (("dtype", 3, -6), ("taps", 1, -6), ("steps", 0, -3), ("n", -1, -3), ("weight", None, -1), ("x", p + 2, -2), ("y", None, -1)):
        bad = cx.ConvArgs.from_buffer_copy(conv)
        setattr(bad, field, value)
        assert lib.craftax_causal_conv(bad, None) == code, field
        assert lib.craftax_last_error()
    back = cx.ConvArgs.from_buffer_copy(conv)
    back.dy = back.dx = p
    back.dweight = p
    need = lib.craftax_causal_conv_workspace_bytes(back)
    assert need > 0 and lib.craftax_causal_conv_backward(back, None) == -1
    work = torch.zeros(need, dtype=torch.uint8, device="cuda")
    back.workspace, back.workspace_bytes = work.data_ptr(), need - 1
    assert lib.craftax_causal_conv_backward(back, None) == -3
    back.workspace, back.workspace_bytes = work.data_ptr() + 4, need
    assert lib.craftax_causal_conv_backward(back, None) == -2
    scan = cx.ScanArgs(dtype=0, steps=1, n=1, channels=2, states=8, groups=1, a=p, x=p, delta=p, b=p, c=p, y=p)
    assert lib.craftax_selective_scan(scan, None) == 0
    for field, value, code in (("states", 12, -6), ("groups", 0, -3), ("groups", 3, -3), ("a", p + 4, -2), ("state_in", p + 8, -2), ("b", None, -1), ("saved", p + 16, -2)):
        bad = cx.ScanArgs.from_buffer_copy(scan)
        setattr(bad, field, value)
        assert lib.craftax_selective_scan(bad, None) == code, field
    assert lib.craftax_selective_scan_saved_bytes(cx.ScanArgs()) == 0 and lib.craftax_selective_scan_workspace_bytes(cx.ScanArgs(), 1) == 0
    assert lib.craftax_selective_scan_backward(scan, None) == -1 and b"saved" in lib.craftax_last_error()
    norm = cx.NormArgs(dtype=1, residual_dtype=1, steps=1, n=1, channels=4, eps=1e-6, y=p, residual=p, out=p, u=p)
    assert lib.craftax_residual_norm(norm, None) == 0
    for field, value, code in (("residual_dtype", 2, -6), ("gate_act", 3, -6), ("eps", float("nan"), -6), ("channels", 8193, -3), ("u", p + 1, -2), ("out", None, -1)):
        bad = cx.NormArgs.from_buffer_copy(norm)
        setattr(bad, field, value)
        assert lib.craftax_residual_norm(bad, None) == code, field
    torch.cuda.synchronize()
    assert ctypes.sizeof(cx.ConvArgs) == 232
