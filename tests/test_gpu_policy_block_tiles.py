"""Ways through the kernels of the projection and the recurrence that few sizes take: large tiles one behind the other that begin with their bias, every
activation in either size of tile, sequences that a thread goes through in turn."""
import pytest
import torch

import policy_block_reference as ref
import test_gpu_policy_block as block
from memory_reference import gradients
from test_gpu_memory import TYPES, Source, close, plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mem():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2402_16801_amd import memory
    return memory


def _whole(gen, most, *shape):
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").double()


# 66,000 x 512 onto 1,024: 1,032 tiles of 256 x 256, four or five to a block.  4,096 rows: 256 tiles of 128 x 128.
@pytest.mark.parametrize("rows", [66000, 4096])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu_tanh"])
@pytest.mark.parametrize("dtype,residual", [("bf16", None), ("bf16", "same"), ("f16", "f32")])
def test_projection_in_tiles_that_go_on_with_their_bias(mem, rows, act, dtype, residual):
    """Whole numbers, all rows different from 0: pre is exact, and so is out without a bent activation; else it is off by a rounding and by what a
    float32 activation is (some eight roundings of its argument and value)."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    kind, I, O = TYPES[dtype], 512, 1024
    x, w, b, d = _whole(gen, 2, rows, I), _whole(gen, 1, O, I), _whole(gen, 30, O), _whole(gen, 1, rows, O)
    x[:, 0] += 5.0 * (x[:, 0] == 0)
    wide = {None: None, "same": kind, "f32": torch.float32}[residual]
    res = None if wide is None else _whole(gen, 30, rows, O)
    gx, gw, gb, gres = x.to(kind), w.to(kind), b.float(), None if res is None else res.to(wide)
    want_pre = x @ w.t() + b
    want = ref.act(want_pre, act)
    if res is not None:
        want = want + res
    for save in (False, True):
        out, pre = mem.projection(gx, gw, gb, residual=gres, act=act, save=save)
        if save:
            assert torch.equal(pre, want_pre.to(kind))
        if act in ("none", "relu"):
            assert torch.equal(out, want.to(wide or kind))
        else:
            slack = 2.0 ** -21 * (want_pre.abs() + want.abs()) + 2.0 ** -25
            off = (out.double() - want).abs() - (block.ROUND[out.dtype] * (want.abs() + slack) + slack)
            assert bool((off <= 0).all()), float(off.max())
    if act != "none":
        return
    gd = d.to(wide or kind)
    g = mem.projection_backward(gd, gx, gw, gb, float_weight=True)
    assert torch.equal(g.x, (d @ w).to(kind))
    assert torch.equal(g.weight.double(), d.t() @ x) and torch.equal(g.bias.double(), d.sum(0))


@pytest.mark.parametrize("dtype,ragged", [("bf16", True), ("f32", False)])
def test_recurrence_of_more_environments_than_blocks_are_for(mem, dtype, ragged):
    """512 channels, two to a thread: 1,250 rows of blocks are needed and 1,024 launched, so threads go on to further sequences with the gradients of the
    rates that they have."""
    block.test_recurrence_of_many_environments(mem, dtype, 9, 5000, 512, ragged)


def test_recurrence_of_one_channel_and_more_environments_than_blocks_are_for(mem):
    """One channel, a thread to a sequence: 4,688 blocks are needed and 4,096 launched."""
    T, n = 3, 1200000
    src = Source(n, torch.float32)
    t = block.rec_inputs(src, T, n, 1, True, True)
    first, dy, dstate = src.flags(T, n, 0.2), src.seq(T, n, 1), src.normal(n, 1)
    lengths = (torch.arange(n, dtype=torch.int32) * 7) % (T + 1)
    (y, h), want = gradients(ref.recurrence, t, (dy, dstate), first=first, lengths=lengths)
    args, how = block.rec_args(block.rec_gpu(src, t))
    how.update(first=first.cuda(), lengths=lengths.cuda())
    got_y, got_h, saved = mem.gated_recurrence(*args, save=True, **how)
    close("y", got_y, y, T)
    close("state", got_h, h, T)
    got = mem.gated_recurrence_backward(src.gpu(dy), saved, *args, dstate=plain(dstate), **how)
    for name, value in got._asdict().items():
        close("gradient of " + name, value, want[name], T * n if name == "rate" else T)


def test_projection_of_more_tiles_than_blocks_are_launched(mem):
    """2,097,199 tiles of 128 x 128, 2^21 blocks: the first ones go on to a second tile.  Whole numbers, every value checked."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows, I, O = (2 ** 21 + 47) * 128 - 37, 8, 72
    x = torch.randint(-2, 3, (rows, I), generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    w, b = _whole(gen, 2, O, I), _whole(gen, 9, O)
    out, _ = mem.projection(x, w.to(torch.bfloat16), b.float(), act="relu")
    for at in range(0, rows, 2 ** 24):
        want = torch.relu(x[at:at + 2 ** 24].float() @ w.float().t() + b.float())
        assert torch.equal(out[at:at + 2 ** 24].float(), want), at
