"""Long sequences on few heads, which dl_prefill walks in segments that it joins afterwards: the
64-bit recurrence again, and what an edge between two segments could get wrong."""

import pytest
import torch

import prefill_harness as P
import sequence_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(64, 64), (128, 128), (64, 128), (128, 64)]


def run(op, lens, H, dk, dv, dtype=F32, state="f32", zero_start=False, **kw):
    x = R.inputs(op, lens, H, dk, dv, dtype, BF16 if state == "bf16" else F32, **kw)
    want = R.expected(op, x, grads=False, zero_start=zero_start)
    c = P.Call(op, x, state, zero_start=zero_start)
    c.build()
    c.forward()
    P.check_forward(c, want)
    assert c.tables.err.item() == 0
    return c


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_shapes(op, dk, dv):
    run(op, [1600], 2, dk, dv, seed=1)
    run(op, [1537], 1, dk, dv, BF16, "bf16", seed=2)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("lens", [[3200, 0, 1500], [1, 3150], [1024, 4000, 513, 512, 1632]], ids=str)
def test_ragged(op, lens):
    """Segments of 16 chunks here: sequences of none, of one, of whole and of broken ones."""
    run(op, lens, 1, 64, 64, BF16, seed=3, B=len(lens) + 2, spare=40)


@pytest.mark.parametrize("op", R.OPS)
def test_zero_start(op):
    run(op, [2100], 3, 64, 64, zero_start=True, seed=4)


@pytest.mark.parametrize("op", ["gdn", "kda", "rwkv6", "gla"])
@pytest.mark.parametrize("decay", [0.0, 8.0, 200.0])
def test_decays_from_none_to_everything(op, decay):
    run(op, [1700], 2, 64, 64, seed=5, decay=decay)


@pytest.mark.parametrize("op", R.OPS)
def test_in_two_calls(op):
    """Cut where no segment ends, with the state handed on in place."""
    x = R.inputs(op, [3300], 2, 64, 64, F32, F32, seed=6, B=1)
    whole = P.Call(op, x)
    whole.build()
    whole.forward()
    S, o, cut = x["S"].cuda(), [], 1650
    for a, b in ((0, cut), (cut, 3300)):
        part = dict(x, lens=[b - a], **{k: x[k][a:b].contiguous() for k in ("q", "k", "v", "lam", "beta", "do")
                                        if torch.is_tensor(x[k]) and x[k].shape[0] == 3300})
        c = P.Call(op, part)
        c.S_in = c.S_out = S
        c.build()
        c.forward()
        o.append(c.o)
    assert R.rel(torch.cat(o), whole.o.double().cpu()) <= R.tol(F32)
    assert R.rel(S, whole.S_out.double().cpu()) <= R.tol(F32)


@pytest.mark.parametrize("op", ["gdn", "rwkv6"])
def test_replays(op):
    """A captured call gives the eager call's bits, whatever the workspace holds by then."""
    x = R.inputs(op, [1600, 3100], 1, 64, 128, BF16, F32, seed=7, B=3)
    c = P.Call(op, x)
    c.build()
    c.forward()
    o, S = c.o.clone(), c.S_out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.build()
        c.forward()
    for _ in range(3):
        c.ws.fill_(0xff)
        c.o.fill_(7.0)
        c.S_out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.o, o) and torch.equal(c.S_out, S)


@pytest.mark.parametrize("op", ["gdn", "kda", "gla"])
def test_a_nan_stays_in_its_sequence(op):
    x = R.inputs(op, [1600, 3100], 2, 64, 64, F32, F32, seed=8)
    clean = P.Call(op, x)
    clean.build()
    clean.forward()
    x["v"] = x["v"].clone()
    x["v"][700, 0, 3] = float("nan")
    c = P.Call(op, x)
    c.build()
    c.forward()
    a, b = x["slots"]
    assert torch.equal(c.o[1600:], clean.o[1600:]) and torch.equal(c.S_out[b], clean.S_out[b])
    assert torch.equal(c.o[:672], clean.o[:672]) and torch.equal(c.o[:1600, 1], clean.o[:1600, 1])
    assert torch.isnan(c.o[700:1600, 0, 3]).all() and torch.isnan(c.S_out[a, 0, :, 3]).all()


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("state", ["f32", "bf16"])
def test_in_place(op, state):
    """The last segment writes the state that the first one reads: the same bits as apart."""
    x = R.inputs(op, [1600, 31, 5000], 3, 64, 64, BF16, BF16 if state == "bf16" else F32, seed=9)
    c = P.Call(op, x, state)
    c.build()
    c.forward()
    o, S = c.o.clone(), c.S_out.clone()
    c.S_in = c.S_out = x["S"].cuda()
    c.forward()
    assert torch.equal(c.o, o) and torch.equal(c.S_out, S)
