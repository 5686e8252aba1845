"""Whole sequences on the GPU against the 64-bit recurrence: every operator, head shape and
type, lengths around the chunk's edges, empty sequences, spare rows, strong decays."""

import pytest
import torch

import prefill_harness as P
import sequence_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(64, 64), (128, 128), (64, 128), (128, 64)]
LENS = [[1], [31, 32, 33], [0, 5, 0, 1], [16, 15, 17, 48], [64, 65, 0, 1, 97]]


def run(op, lens, H, dk, dv, dtype=F32, state="f32", backward=False, zero_start=False, **kw):
    st = BF16 if state == "bf16" else F32
    x = R.inputs(op, lens, H, dk, dv, dtype, st, **kw)
    want = R.expected(op, x, grads=backward, zero_start=zero_start)
    c = P.Call(op, x, state, backward, zero_start)
    c.build()
    c.forward()
    P.check_forward(c, want)
    if backward:
        c.backward()
        P.check_grads(c, want, strong=kw.get("decay", 1.0) > 1.0)
    assert c.tables.err.item() == 0
    return c


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_forward_shapes(op, dk, dv):
    run(op, [40, 3], 2, dk, dv, seed=1)
    run(op, [40, 3], 2, dk, dv, BF16, seed=2)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_forward_lengths(op, lens):
    run(op, lens, 3, 64, 64, seed=4, B=len(lens) + 2, spare=9)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_backward_shapes(op, dk, dv):
    run(op, [40, 3], 2, dk, dv, backward=True, seed=1)
    run(op, [40, 3], 2, dk, dv, BF16, backward=True, seed=2)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_backward_lengths(op, lens):
    run(op, lens, 3, 64, 64, backward=True, seed=4, B=len(lens) + 2, spare=9)


@pytest.mark.parametrize("op", R.OPS)
def test_bf16_state(op):
    run(op, [33, 0, 70], 2, 64, 128, BF16, "bf16", backward=True, seed=6)


@pytest.mark.parametrize("op", R.OPS)
def test_zero_start(op):
    run(op, [33, 2], 2, 128, 64, backward=True, zero_start=True, seed=7)


@pytest.mark.parametrize("op", ["gdn", "kda", "rwkv6", "gla"])
@pytest.mark.parametrize("decay", [0.0, 8.0, 200.0])
def test_decays_from_none_to_everything(op, decay):
    """Log-decays scaled up to sums far past what a factor e^(l_i) e^(-l_j) could hold."""
    run(op, [70, 20], 2, 64, 64, backward=True, seed=8, decay=decay)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_many_heads(op, dk, dv):
    """Enough (sequence, head) pairs for workgroups that walk whole heads."""
    dtype = BF16 if dk == dv else F32
    run(op, [37, 5, 64], 1024 // (dv // 32) // 3 + 1, dk, dv, dtype, backward=True, seed=9)
