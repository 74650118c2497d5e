"""The policy memory operators refuse what is not on a GPU, and their structures match the C header's (no GPU needed)."""
import ctypes
import importlib.util
import os
import subprocess

import pytest
import torch

from paper_2402_16801_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mem():
    from paper_2402_16801_amd import memory
    return memory


def test_tensors_on_the_cpu_are_refused(mem):
    x, state = torch.zeros(2, 3, 8), torch.zeros(3, 3, 8)
    with pytest.raises(binding.CraftaxError):
        mem.causal_conv(x, torch.zeros(8, 4))
    with pytest.raises(binding.CraftaxError):
        mem.causal_conv_step(x[0], torch.zeros(8, 4), None, state)
    with pytest.raises(binding.CraftaxError):
        mem.selective_scan(x, x, torch.zeros(8, 16), torch.zeros(2, 3, 1, 16), torch.zeros(2, 3, 1, 16))
    with pytest.raises(binding.CraftaxError):
        mem.residual_norm(x, x)


def test_an_unknown_gate_is_refused(mem):
    with pytest.raises(binding.CraftaxError, match="gate_act"):
        mem.residual_norm(torch.zeros(1, 1, 8), torch.zeros(1, 1, 8), gate_act="tanh")


def test_counts_that_32_bits_do_not_hold_with_what_is_read_ahead_are_refused():
    """At the C entry, before anything is looked at on a device: the addresses are none."""
    lib, at, most = binding.load(), 1 << 20, 2 ** 31 - 4096
    conv = dict(dtype=1, n=1, channels=1, taps=2, weight=at, x=at, y=at, dy=at, dx=at)
    scan = dict(dtype=1, n=1, channels=1, states=8, groups=1, a=at, x=at, delta=at, b=at, c=at, y=at, dy=at, dx=at, ddelta=at, db=at, dc=at, da=at, saved=at)
    for args, calls in ((binding.ConvArgs(steps=most + 1, **conv), ("causal_conv", "causal_conv_backward")),
                        (binding.ScanArgs(steps=most + 1, **scan), ("selective_scan", "selective_scan_backward"))):
        for call in calls:
            assert getattr(lib, "craftax_" + call)(args, None) == -3 and b"steps" in lib.craftax_last_error(), call
        args.steps, args.n = 1, most + 1
        for call in calls:
            assert getattr(lib, "craftax_" + call)(args, None) == -3 and b"n * channels" in lib.craftax_last_error(), call


def test_structures_match_the_header(tmp_path):
    pairs = [("craftax_conv_args", binding.ConvArgs), ("craftax_scan_args", binding.ScanArgs),
             ("craftax_norm_args", binding.NormArgs)]
    lines, want = [], []
    for name, struct in pairs:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(struct))
        fields = [field[0] for field in struct._fields_]
        for field in fields:
            base, _, last = field.rpartition("_")          # a view's members lie side by side: x, x_step, x_env
            member = f"{base}.{last}" if last in ("step", "env") and base in fields else field
            lines.append(f'printf("%zu\\n", offsetof({name}, {member}));')
            want.append(getattr(struct, field).offset)
    source = tmp_path / "sizes.c"
    source.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "craftax.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "sizes"), str(source)], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in got] == want


def test_the_returns_of_the_example_go_on_behind_the_rollout():
    """The return of the last step: its reward and the discounted value of what followed it, nothing where the episode ended."""
    spec = importlib.util.spec_from_file_location("policy_memory", os.path.join(ROOT, "examples", "policy_memory.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    reward = torch.tensor([[1.0, 0.0, 2.0], [0.5, 1.0, 0.0], [0.25, 2.0, 1.0]], dtype=torch.float64)
    done = torch.tensor([[0, 1, 0], [0, 0, 0], [0, 0, 1]], dtype=torch.uint8)
    values = torch.tensor([[0.5, 1.5, -1.0], [2.0, 0.0, 1.0], [3.0, -2.0, 4.0]], dtype=torch.float64)
    logits = torch.zeros(3, 3, example.ACTIONS, dtype=torch.float64)
    seen = {"obs": None, "first": None, "reward": reward, "done": done, "actions": torch.zeros(3, 3, dtype=torch.int32),
            "ahead": torch.tensor([8.0, -16.0, 32.0], dtype=torch.float64)}
    loss, _ = example.loss_of(lambda obs, states, first: (logits, values, None), seen, None, discount=0.5)
    returns = torch.tensor([[1 + 0.25 + 0.0625 + 1.0, 0.0, 2 + 0.0 + 0.25], [0.5 + 0.125 + 2.0, 1 + 1.0 - 4.0, 0.5], [0.25 + 4.0, 2.0 - 8.0, 1.0]], dtype=torch.float64)
    chance = torch.tensor(1.0 / example.ACTIONS, dtype=torch.float64)
    want = -(chance.log() * (returns - values)).mean() + 0.5 * (returns - values).square().mean() + 0.01 * chance.log()
    assert abs(float(loss - want)) <= 1e-12


def test_quick_builds_compile_what_has_changed(monkeypatch):
    """only_changed: neither the extension nor, behind a change of the extension's source, the kernels are compiled again."""
    from paper_2402_16801_amd import build
    ran = []

    class Done:
        returncode, stderr = 0, ""

    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **how: ran.append(cmd) or Done())
    monkeypatch.setattr(build.os, "makedirs", lambda *a, **k: None)
    exists, getmtime, age = os.path.exists, os.path.getmtime, {".cpp": 3, ".o": 2, ".so": 4}              # everything else of the repository: 1

    def ours(p):
        return str(p).startswith(ROOT)

    monkeypatch.setattr(build.os.path, "exists", lambda p: ours(p) or exists(p))
    monkeypatch.setattr(build.os.path, "getmtime", lambda p: age.get(os.path.splitext(p)[1], 1) if ours(p) else getmtime(p))
    build.build_all(only_changed=True)
    assert len(ran) == 2 and all("-c" not in cmd for cmd in ran)           # the two libraries are linked
    del ran[:]
    age[".so"] = 2
    build.build_all(only_changed=True)
    assert len(ran) == 3 and sum(build.MARSHAL_SRC in cmd for cmd in ran) == 1
