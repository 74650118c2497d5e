"""The gated recurrence, the projection and the dropout: structures as in the C header, refusals that need no GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

import policy_block_reference as ref
from paper_2402_16801_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mem():
    from paper_2402_16801_amd import memory
    return memory


def test_tensors_on_the_cpu_are_refused(mem):
    x = torch.zeros(2, 3, 8)
    for call in (lambda: mem.gated_recurrence(x, x, x, torch.zeros(8)), lambda: mem.gated_recurrence_step(x[0], x[0], x[0], torch.zeros(8), torch.zeros(3, 8)),
                 lambda: mem.projection(x, torch.zeros(4, 8)), lambda: mem.projection_backward(x, x, torch.zeros(8, 8)), lambda: mem.residual_dropout(x, 0.5, 1)):
        with pytest.raises(binding.CraftaxError, match="no CPU path"):
            call()
    with pytest.raises(binding.CraftaxError, match="act must be"):
        mem.projection(x, torch.zeros(4, 8), act="tanh")
    with pytest.raises(binding.CraftaxError, match="activations must be"):
        mem.residual_dropout_backward(x, 0.5, 1, dtype=torch.int32)


def test_counts_out_of_range_are_refused_at_the_c_entry():
    """Before anything is looked at on a device: the addresses are none."""
    lib, at, most = binding.load(), 1 << 20, 2 ** 31 - 4096
    rec = binding.RecurrenceArgs(dtype=1, steps=most + 1, n=1, channels=1, rate=at, x=at, decay=at, intake=at, y=at, saved=at, dy=at, dx=at, ddecay=at, dintake=at)
    for call in (lib.craftax_gated_recurrence, lib.craftax_gated_recurrence_backward):
        rec.steps, rec.n = most + 1, 1
        assert call(rec, None) == -3 and b"steps" in lib.craftax_last_error()
        rec.steps, rec.n = 1, most + 1
        assert call(rec, None) == -3 and b"n * channels" in lib.craftax_last_error()
    pro = binding.ProjectionArgs(dtype=1, out_dtype=1, steps=1 << 16, n=1 << 15, inputs=1, outputs=1, weight=at, weight_row=1, weight_column=1, x=at, out=at, dout=at)
    for call in (lib.craftax_projection, lib.craftax_projection_backward):
        assert call(pro, None) == -3 and b"steps * n" in lib.craftax_last_error()
    for steps, n, inputs, outputs in ((1 << 15, 1 << 15, 1 << 13, 1), (1, 1, 1 << 30, 1 << 13), (1 << 20, 1 << 10, 1, most)):
        pro.steps, pro.n, pro.inputs, pro.outputs = steps, n, inputs, outputs
        for backward, call in enumerate((lib.craftax_projection, lib.craftax_projection_backward)):
            assert call(pro, None) == -3 and b"memory" in lib.craftax_last_error()
            assert lib.craftax_projection_workspace_bytes(pro, backward) == 0
    drop = binding.DropoutArgs(dtype=1, out_dtype=1, steps=1 << 16, n=1 << 15, channels=1, p=0.5, x=at, out=at)
    assert lib.craftax_residual_dropout(drop, None) == -3 and b"steps * n" in lib.craftax_last_error()


def test_structures_match_the_header(tmp_path):
    pairs = [("craftax_recurrence_args", binding.RecurrenceArgs), ("craftax_projection_args", binding.ProjectionArgs), ("craftax_dropout_args", binding.DropoutArgs)]
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
    text = open(os.path.join(ROOT, "include", "craftax.h")).read()
    for k, name in enumerate(("NONE", "RELU", "SILU", "GELU_TANH")):
        assert f"CRAFTAX_ACT_{name} = {k}" in text and getattr(binding, "ACT_" + name) == k


def test_the_plain_generator_gives_the_published_numbers():
    """Philox4x32-10 of the published test: counter and key of ones and of zeros."""
    for word, numbers in ((0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)), (0xFFFFFFFF, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD))):
        seed, step = word | word << 32, word | word << 32
        lowest = [n >> (16 * h) & 0xFFFF for n in numbers for h in (0, 1)]
        # the mask at thresholds next to each number says the number
        for j, n in enumerate(lowest):
            block = word
            for p, kept in ((n / 65536, True), ((n + 1) / 65536, False)):
                assert bool(_one(seed, step, block, p)[j]) == kept


def _one(seed, step, word, p):
    """The eight truth values of the counter (word, word, step)."""
    import numpy as np
    c, k = [word, word, step & 0xFFFFFFFF, step >> 32], [seed & 0xFFFFFFFF, seed >> 32]
    if word == 0:
        return ref.keep_mask(seed, step, 0, 1, 1, 8, p)[0][0, 0]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.array([(c[j // 2] >> (16 * (j % 2)) & 0xFFFF) >= int(p * 65536 + 0.5) for j in range(8)])
