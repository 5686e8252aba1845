"""What whole-sequence calls make of values that a program has by choice or by accident: outputs
rounded once."""

import pytest
import torch

import prefill_harness as P
import sequence_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(64, 64), (128, 128), (64, 128), (128, 64)]


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
@pytest.mark.parametrize("lens", [[70, 33], [1600]], ids=str)
def test_bf16_outputs_are_rounded_once(op, dk, dv, lens):
    """Every bf16 output is within half a step of the exact value, and what fp32 arithmetic adds:
    TOL_F32 of the outputs' size, of which an element's own error is a share that no more than
    a few of its head's 64 or 128 columns can exceed four times."""
    x = R.inputs(op, lens, 2, dk, dv, BF16, F32, seed=1)
    want = R.expected(op, x)["o"]
    c = P.Call(op, x)
    c.build()
    c.forward()
    size = (want ** 2).mean(-1, keepdim=True).sqrt()
    slack = (c.o.double().cpu() - want).abs() - torch.finfo(BF16).eps / 2 * want.abs()
    assert (slack / size).max().item() <= 4 * R.TOL_F32
