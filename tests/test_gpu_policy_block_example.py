"""The example's policy with a gated recurrence: acting and learning are the same policy, dropout and all, and its gradients are the definition's.

Tolerances as in test_gpu_policy_memory.py: some ten roundings of the type for logits and states, 16 * 32 * 2^-24 * sqrt(1400) of a tensor's largest
gradient for about eight sums one behind the other, forward and backward.
"""
import copy
import importlib.util
import os
import types

import pytest
import torch

import memory_reference as older
import policy_block_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("policy_memory", os.path.join(ROOT, "examples", "policy_memory.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rollout(example, dtype, n, steps):
    from paper_2402_16801_amd import binding as cx, synth
    torch.manual_seed(5)
    sim = cx.Craftax(n, cx.default_config(obs_mode=cx.OBS_SYM_F32, max_episode_steps=15))
    sim.reset(synth.seeds_for(n))
    policy = example.Policy(sim.obs_bytes // 4, width=64, dtype=dtype, cell="recurrence", drop=0.25)
    states, first = policy.empty(n), torch.ones(n, dtype=torch.uint8, device="cuda")
    example.act(policy, sim, states, first, 11)
    began = [[v.clone() for v in state] for state in states]
    seen = example.act(policy, sim, states, first, steps)
    sim.close()
    return policy, began, seen, states


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_acting_and_learning_see_the_same_policy(example, dtype):
    policy, began, seen, states = rollout(example, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], 300, 40)
    assert int(seen["first"][1:].sum()) >= 300 and [int(s[2]) for s in began + states] == [11, 11, 51, 51]
    with torch.no_grad():
        logits, _, after = policy(seen["obs"], began, seen["first"])
    unit = 16 * 2.0 ** (-8 if dtype == "bf16" else -20)
    assert float((logits - seen["logits"]).abs().max()) <= unit * float(logits.abs().max())
    for got, want in zip(after, states):
        for a, b in zip(got, want):
            assert float((a.float() - b.float()).abs().max()) <= unit * float(b.float().abs().max())


def test_the_update_against_64_bits(example, monkeypatch):
    policy, began, seen, _ = rollout(example, torch.float32, 40, 24)
    loss, _ = example.loss_of(policy, seen, began)
    loss.backward()
    plain = copy.deepcopy(policy).cpu().double()
    plain.dtype = torch.float64

    def dropout(x, p, seed, *, residual, step):
        keep, scale = ref.keep_mask(seed, int(step), 0, *x.shape, p)
        return ref.dropout(x, keep, scale, residual)

    def project(x, weight, bias=None):
        return ref.project(x, weight, bias)[0]

    monkeypatch.setattr(example, "memory", types.SimpleNamespace(conv=older.conv, norm=older.norm, recurrence=ref.recurrence, project=project, dropout=dropout))
    plain_loss, _ = example.loss_of(plain, {k: v.cpu() if v.dtype != torch.float32 else v.cpu().double() for k, v in seen.items()},
                                    [[v.cpu() if v.dtype == torch.int64 else v.cpu().double() for v in state] for state in began])
    for p in plain.parameters():
        p.grad = None
    plain_loss.backward()
    assert abs(loss.item() - plain_loss.item()) <= 1.1e-3 * max(1.0, abs(plain_loss.item()))
    for (name, got), (_, want) in zip(policy.named_parameters(), plain.named_parameters()):
        big = float(want.grad.abs().max())
        assert big > 0, name
        off = float((got.grad.cpu().double() - want.grad).abs().max())
        assert off <= 1.1e-3 * big, f"{name}: {off:.3g} of {big:.3g}"


def test_the_example_runs(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["policy_memory.py", "--envs", "257", "--steps", "9", "--updates", "2", "--cell", "recurrence"])
    example.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and all("nan" not in v and "inf" not in v for v in lines)
