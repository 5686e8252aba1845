"""Whole-sequence calls without a token row: states pass through, and their gradients."""

import pytest
import torch

import sequence_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("op", R.OPS)
def test_scan_without_rows(op):
    from paper_2608_15533_amd.sequence import delta_scan
    x = R.inputs(op, [0, 0], 2, 64, 128, seed=1)
    y = {n: x[n].cuda().requires_grad_() for n in R.GRADS if x[n] is not None}
    o, S = delta_scan(op, y["q"], y["k"], y["v"], y.get("lam"), y.get("beta"), y.get("u"), y["S"],
                      torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert o.shape == (0, 2, 128) and torch.equal(S, y["S"])
    got = torch.autograd.grad((S * x["dS"].cuda()).sum(), list(y.values()))
    for (name, leaf), g in zip(y.items(), got):
        want = x["dS"].cuda() if name == "S" else torch.zeros_like(leaf)
        assert torch.equal(g, want), name


def test_engine_prompts_without_tokens():
    """A slot taken without a token starts from zero; an active one keeps its state."""
    from paper_2608_15533_amd import decode, deltalog as D
    desc = D.make_desc("gla", 3, 2, 64, 64, 4, "f32")
    eng = decode.DecodeEngine(desc, 1)
    eng.states[0].S.fill_(3.0)
    empty = [[None if t is None else t.cuda() for t in (x["q"], x["k"], x["v"], x["lam"], x["beta"])]
             for x in [R.inputs("gla", [], 2, 64, 64, B=1)]]
    slots, outs = eng.prefill([0, 0], empty)
    assert len(slots) == 2 and outs[0].shape == (0, 2, 64)
    assert torch.all(eng.states[0].S[slots] == 0)
    eng.states[0].S.fill_(3.0)
    assert eng.prefill([0], empty, slots=slots[:1])[0] == slots[:1]
    assert torch.all(eng.states[0].S == 3.0)
