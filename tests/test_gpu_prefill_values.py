"""What whole-sequence calls make of values that a program has by choice or by accident: fp32
inputs, bf16 outputs rounded once, log-decays that are not a number or above zero."""

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


# fp32 all the way: a sum of up to 128 + 32 terms rounds as often, each time by 2^-24 / sqrt(3) of what
# it holds (root mean square), so it is off by sqrt(160) of that, 4.4e-7; five such products in a row by
# sqrt(5) times as much, 1e-6; an exponential adds 2^-23 (its last bit).  Twice that.
FULL = 2e-6


def check_full(c, want, backward):
    lens, slots = sum(c.x["lens"]), c.x["slots"]
    pairs = [("o", c.o[:lens], want["o"]), ("S", c.S_out[slots], want["S"][slots])]
    for name, ref in want.get("grads", {}).items() if backward else ():
        got = getattr(c.grads, name)
        if name == "dS":
            got, ref = got[slots], ref[slots]
        elif name != "du":
            got = got[:lens]
        pairs.append((name, got, ref))
    errors = {name: R.rel(got, ref) for name, got, ref in pairs}
    assert max(errors.values()) <= FULL, errors


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_fp32_inputs_keep_fp32(op, dk, dv):
    x = R.inputs(op, [150, 0, 33], 3, dk, dv, F32, F32, seed=4)
    want = R.expected(op, x, grads=True)
    c = P.Call(op, x, backward=True)
    c.build()
    c.forward()
    c.backward()
    check_full(c, want, True)


@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_bf16_inputs_have_fp32_states_and_gate_gradients(op, dk, dv):
    """What is fp32 of a call with bf16 inputs is as good as with fp32 ones."""
    for lens, H, backward in (([150, 0, 33], 3, True), ([1650, 40], 2, False), ([33, 40], 130, True)):
        x = R.inputs(op, lens, H, dk, dv, BF16, F32, seed=6)
        want = R.expected(op, x, grads=backward)
        c = P.Call(op, x, backward=backward)
        c.build()
        c.forward()
        slots = x["slots"]
        errors = {"S": R.rel(c.S_out[slots], want["S"][slots])}
        if backward:
            c.backward()
            errors["dS"] = R.rel(c.grads.dS[slots], want["grads"]["dS"][slots])
            for name in ("dlam", "dbeta", "du"):
                if name in want["grads"]:
                    got = getattr(c.grads, name)
                    errors[name] = R.rel(got, want["grads"][name])
        assert max(errors.values()) <= FULL, errors


@pytest.mark.parametrize("op", R.OPS)
def test_fp32_inputs_keep_fp32_over_segments(op):
    x = R.inputs(op, [1700, 40], 2, 128, 64, F32, F32, seed=5)
    want = R.expected(op, x)
    c = P.Call(op, x)
    c.build()
    c.forward()
    check_full(c, want, False)


@pytest.mark.parametrize("op", [o for o in R.OPS if o != "linattn"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("at", [0, 7, 20, 31, 32, 39])
def test_a_log_decay_that_is_not_a_number(op, dtype, at):
    """It makes its head's state one from its token on: the sequence's later outputs, its final state
    and what flows back through it; other heads and sequences keep their bits."""
    lens, H = [40, 40, 40], 3
    x = R.inputs(op, lens, H, 64, 64, dtype, seed=2)
    c = P.Call(op, x, backward=True)
    c.build()
    c.forward()
    c.backward()
    results = lambda: [t for t in (c.o, c.S_out, c.grads.dq, c.grads.dk, c.grads.dv,  # noqa: E731
                                   c.grads.dlam, c.grads.dS) if t is not None]
    clean = [t.clone() for t in results()]
    per_key = c.x["lam"].dim() == 3
    if per_key:
        c.x["lam"][40 + at, 1, 5] = float("nan")
    else:
        c.x["lam"][40 + at, 1] = float("nan")
    c.forward()
    c.backward()
    mid = x["slots"][1]
    first = 40 + at + (op == "rwkv6")                # reads the state before its token
    assert torch.isnan(c.o[first:80, 1]).all()
    row = c.S_out[mid, 1, 5] if per_key else c.S_out[mid, 1]
    assert torch.isnan(row).all()
    row = c.grads.dS[mid, 1, 5] if per_key else c.grads.dS[mid, 1]
    assert torch.isnan(row).all()
    lam = c.grads.dlam[40:40 + at + 1, 1]
    assert torch.isnan(lam[..., 5] if per_key else lam).all()
    for a, b in zip(clean, results()):
        a, b = a.clone(), b.clone()
        if a.dim() == 4:
            a[mid, 1] = b[mid, 1] = 0
        else:
            a[40:80, 1] = b[40:80, 1] = 0
        assert torch.equal(a, b)


@pytest.mark.parametrize("op", [o for o in R.OPS if o != "linattn"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_log_decays_above_zero(op, dtype):
    """Outside the domain, as for the decode step, which takes them at their value: so do these."""
    x = R.inputs(op, [70, 20], 2, 64, 64, dtype, seed=3)
    x["lam"] = x["lam"].clone()
    x["lam"][::3] = 0.125
    want = R.expected(op, x, grads=True)
    c = P.Call(op, x, backward=True)
    c.build()
    c.forward()
    c.backward()
    P.check_forward(c, want)
    P.check_grads(c, want)
