"""Every build of the whole-sequence walks, in both types: (sequence, head) pairs on both sides of
what picks workgroups of two, four and eight waves, judged head by head."""

import pytest
import torch

import prefill_harness as P
import sequence_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(64, 64), (128, 128), (64, 128), (128, 64)]


def _blocks(x, lens):
    """Norms [sequence, head] of packed rows [N,H,...]."""
    return torch.stack([p.flatten(2).norm(dim=(0, 2)) if p.shape[0] else p.new_zeros(p.shape[1])
                        for p in x.reshape(x.shape[0], x.shape[1], -1).split(lens)])


def check_by_head(name, got, ref, lens):
    """The error of every (sequence, head) against a block's size: its own or the usual one of its
    sequence (a block whose terms happen to cancel has the errors of the others).  The bar is that
    of the whole: it is derived product by product, so it holds for every block of rows too."""
    got, ref = got[:sum(lens)].detach(), ref.detach()
    err = _blocks(got.double().cpu() - ref, lens)
    size = _blocks(ref, lens)
    usual = (size ** 2).mean(1, keepdim=True).sqrt()
    bar = R.tol(got.dtype) * (size + usual)
    worst = (err / bar.clamp(min=1e-300)).max().item()
    assert torch.all(err <= bar), f"{name}: {worst:.2e} of the bar"


def run(op, lens, H, dk, dv, dtype, backward=True, state="f32", seed=0, **kw):
    x = R.inputs(op, lens, H, dk, dv, dtype, BF16 if state == "bf16" else F32, seed=seed, **kw)
    want = R.expected(op, x, grads=backward)
    c = P.Call(op, x, state, backward)
    c.build()
    c.forward()
    P.check_forward(c, want)
    check_by_head("o", c.o, want["o"], lens)
    slots = x["slots"]
    one = [1] * len(lens)
    check_by_head("S", c.S_out[slots], want["S"][slots], one)
    if backward:
        c.backward()
        P.check_grads(c, want)
        for name in ("dq", "dk", "dv"):
            check_by_head(name, getattr(c.grads, name), want["grads"][name], lens)
        check_by_head("dS", c.grads.dS[slots], want["grads"]["dS"][slots], one)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
@pytest.mark.parametrize("pairs", [126, 130, 254, 260])
def test_bf16_pairs_around_the_choices(op, dk, dv, pairs):
    """Two sequences of H heads.  For dv = 128 (twice as many pairs for dv = 64) workgroups of two
    waves end at 256 pairs forward and 128 backward with 64 keys, at half of that with 128 and raw
    operands, at a quarter with planes."""
    H = pairs // 2 * (128 // dv)
    run(op, [35, 9], H, dk, dv, BF16, seed=1)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_bf16_whole_heads(op, dk, dv):
    run(op, [37, 5, 64, 0, 33, 1, 40], 40 * (128 // dv), dk, dv, BF16, seed=2, B=9, spare=3)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 64)])
def test_f32_whole_heads(op, dk, dv):
    run(op, [37, 5, 64], 50 * (128 // dv), dk, dv, F32, seed=3)
