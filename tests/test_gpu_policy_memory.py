"""The policy memory operators together (examples/policy_memory.py), and sequences cut into many parts.

Tolerances as in test_gpu_memory.py: an output is rounded once, and a sum of m terms in 32 bits may be off by
32 * 2^-24 * sqrt(m) times the largest value.  A network of two blocks puts about eight such sums (products of
up to 1,400 terms, the scan over the rollout) one behind the other, forward and again backward: 16 * 32 * 2^-24 *
sqrt(1400) = 1.1e-3 of the largest gradient of a tensor.
"""
import copy
import importlib.util
import os
import types

import pytest
import torch

import memory_reference as ref
from test_gpu_memory import TYPES, Source, close, plain, scan_gpu, scan_inputs

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mem():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2402_16801_amd import memory
    return memory


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_memory", os.path.join(ROOT, "examples", "policy_memory.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


# dtype, T, n, D, N, G, order, begins, ragged: few environments of many steps, with a memory of thousands of steps
@pytest.mark.parametrize("case", [
    ("f32", 3001, 1, 64, 16, 1, "time", 0.0, False),
    ("f32", 2050, 2, 40, 32, 1, "batch", 0.002, True),
    ("bf16", 4096, 1, 130, 8, 2, "slice", 0.001, False),
    ("f16", 1200, 3, 64, 16, 2, "time", 0.002, True),
], ids=lambda v: "-".join(str(x) for x in v))
def test_scan_of_many_parts(mem, case):
    dtype, T, n, D, N, G, order, begins, ragged = case
    src = Source(T + D, TYPES[dtype], order)
    t = scan_inputs(src, T, n, D, N, G, True, True)
    t["delta_bias"] -= 4.0                                   # rates of some 0.002 to 0.1 a step
    t["b"] = (t["b"] * 0.125).to(TYPES[dtype]).double()
    first = src.flags(T, n, begins) if begins else None
    lengths = torch.tensor([T - 5, 700, T][:n], dtype=torch.int32) if ragged else None
    dy, dstate = src.seq(T, n, D), src.normal(n, D, N)
    (y, h), want = ref.gradients(ref.scan, t, (dy, dstate), first=first, lengths=lengths)
    g = scan_gpu(src, t)
    how = {k: g[k] for k in ("d", "z", "delta_bias", "state")}
    how["first"] = None if first is None else first.cuda()
    how["lengths"] = None if lengths is None else lengths.cuda()
    args = [g[k] for k in ("x", "delta", "a", "b", "c")]
    chain = N * T
    for save in (False, True):
        got_y, got_h, saved = mem.selective_scan(*args, save=save, **how)
        close("y", got_y, y, chain)
        close("state", got_h, h, chain)
    got = mem.selective_scan_backward(src.gpu(dy), saved, *args, dstate=plain(dstate), **how)
    for name, value in got._asdict().items():
        close("gradient of " + name, value, want[name], chain + D)


@pytest.mark.parametrize("T", [1, 8, 40, 2000])
@pytest.mark.parametrize("operator", ["scan", "conv"])
def test_a_state_is_updated_in_place(mem, operator, T):
    """At the C entry state_out may be state_in, for one part of steps as for many."""
    from paper_2402_16801_amd import binding as cx
    lib, n, D = cx.load(), 2, 66
    src = Source(T, torch.float32)
    seqs = {k: src.gpu(src.seq(T, n, D)) for k in ("x", "y")}
    seqs.update({k: src.gpu(src.seq(T, n, 16)) for k in ("b", "c")})
    views = {f: v for k, t in seqs.items() for f, v in ((k, t.data_ptr()), (k + "_step", t.stride(0)), (k + "_env", t.stride(1)))}
    x = seqs["x"]
    if operator == "scan":
        a, state = -torch.rand(D, 16, device="cuda") * 0.1, torch.randn(n, D, 16, device="cuda")
        want_y, want, _ = mem.selective_scan(x, x, a, seqs["b"].unsqueeze(2), seqs["c"].unsqueeze(2), state=state)
        args = cx.ScanArgs(dtype=0, softplus=1, steps=T, n=n, channels=D, states=16, groups=1, a=a.data_ptr(), delta=x.data_ptr(),
                           delta_step=x.stride(0), delta_env=x.stride(1), state_in=state.data_ptr(), state_out=state.data_ptr(), **views)
        need = lib.craftax_selective_scan_workspace_bytes(args, 0)
        work = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        args.workspace, args.workspace_bytes = work.data_ptr(), need
        call = lib.craftax_selective_scan
    else:
        weight, state = torch.randn(D, 4, device="cuda"), torch.randn(n, 3, D, device="cuda")
        want_y, want = mem.causal_conv(x, weight, state=state)
        args = cx.ConvArgs(dtype=0, silu=1, steps=T, n=n, channels=D, taps=4, weight=weight.data_ptr(), state_in=state.data_ptr(),
                           state_out=state.data_ptr(), **{k: v for k, v in views.items() if k[0] in "xy"})
        call = lib.craftax_causal_conv
    torch.cuda.synchronize()
    assert call(args, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(seqs["y"], want_y) and torch.equal(state, want)


def rollout(example, dtype, n=300, steps=40):
    """A policy and what it saw while episodes of 15 steps end, some of them within the rollout's first steps."""
    from paper_2402_16801_amd import binding as cx, synth
    torch.manual_seed(3)
    sim = cx.Craftax(n, cx.default_config(obs_mode=cx.OBS_SYM_F32, max_episode_steps=15))
    sim.reset(synth.seeds_for(n))
    policy = example.Policy(sim.obs_bytes // 4, width=64, dtype=dtype)
    states, first = policy.empty(n), torch.ones(n, dtype=torch.uint8, device="cuda")
    example.act(policy, sim, states, first, 11)
    began = [[v.clone() for v in state] for state in states]
    seen = example.act(policy, sim, states, first, steps)
    sim.close()
    return policy, began, seen, states


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_acting_and_learning_see_the_same_policy(example, dtype):
    policy, began, seen, states = rollout(example, TYPES[dtype])
    assert int(seen["done"].sum()) >= 2 * 300 and int(seen["first"][1:].sum()) == int(seen["done"][:-1].sum())
    with torch.no_grad():
        logits, _, after = policy(seen["obs"], began, seen["first"])
    # the operators give the same values for a token and for a sequence up to their tolerance; a product may be rounded
    # differently for another number of rows, once per product and block: some ten roundings of the type
    unit = 16 * 2.0 ** (-8 if dtype == "bf16" else -20)
    assert float((logits - seen["logits"]).abs().max()) <= unit * float(logits.abs().max())
    for got, want in zip(after, states):
        for a, b in zip(got, want):
            assert float((a.float() - b.float()).abs().max()) <= unit * float(b.float().abs().max())


def test_the_update_against_64_bits(example, monkeypatch):
    policy, began, seen, _ = rollout(example, torch.float32, n=40, steps=24)
    loss, _ = example.loss_of(policy, seen, began)
    loss.backward()
    plain_policy = copy.deepcopy(policy).cpu().double()
    plain_policy.dtype = torch.float64
    monkeypatch.setattr(example, "memory", types.SimpleNamespace(conv=ref.conv, scan=ref.scan, norm=ref.norm))
    plain_loss, _ = example.loss_of(plain_policy, {k: v.cpu() if v.dtype != torch.float32 else v.cpu().double() for k, v in seen.items()},
                                    [[v.cpu().double() for v in state] for state in began])
    for p in plain_policy.parameters():
        p.grad = None
    plain_loss.backward()
    assert abs(loss.item() - plain_loss.item()) <= 1.1e-3 * max(1.0, abs(plain_loss.item()))
    for (name, got), (_, want) in zip(policy.named_parameters(), plain_policy.named_parameters()):
        big = float(want.grad.abs().max())
        assert big > 0 or "w_scan" in name, name
        off = float((got.grad.cpu().double() - want.grad).abs().max())
        assert off <= 1.1e-3 * big, f"{name}: {off:.3g} of {big:.3g}"


def test_the_example_runs(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["policy_memory.py", "--envs", "257", "--steps", "9", "--updates", "2"])
    example.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and all("nan" not in v and "inf" not in v for v in lines)
