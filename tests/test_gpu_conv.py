"""The short causal convolution against 64 bits: prompts, training, single tokens, as it is used."""

import pytest
import torch

import layer_harness as L
import layer_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])


@TYPES
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("lens,spare,D", [
    ([1], 0, 8), ([2, 0, 1, 3], 0, 64), ([0, 0, 5], 3, 72), ([31, 32, 33, 64, 65], 0, 256),
    ([0], 4, 8), ([100, 3, 0, 130], 5, 520)], ids=str)
def test_sequences(dtype, act, W, lens, spare, D):
    x = R.conv_inputs(lens, D, W, dtype, bias=W != 3, B=len(lens) + 1, seed=W, spare=spare)
    L.check(L.run("conv", x, act), R.conv_expected(x, act))


@TYPES
def test_rows_of_a_wider_tensor(dtype):
    x = R.conv_inputs([40, 7], 136, 4, dtype, seed=1, spare=1)
    L.check(L.run("conv", x, strided=True), R.conv_expected(x))


@TYPES
def test_no_initial_states_and_no_gradient_of_the_final_ones(dtype):
    x = R.conv_inputs([40, 0, 2], 64, 4, dtype, seed=2)
    want = R.conv_expected(x, zero_start=True, final_grad=False)
    L.check(L.run("conv", x, zero_start=True, final_grad=False), want)
    c = L.Packed("conv", x, zero_start=True)
    c.grads = c.D.ConvGrads(c.desc, c.rows)                # and none of the initial states wanted
    c.build()
    c.backward(False)
    want["grads"].pop("s")
    c.forward()
    L.check(c, want)


@pytest.mark.parametrize("n,D", [(400, 64), (3, 12288), (1, 8)])
def test_many_sequences_and_wide_rows(n, D):
    x = R.conv_inputs([(7 * i) % 41 for i in range(n)], D, 4, BF16, seed=3)
    L.check(L.run("conv", x), R.conv_expected(x))


@TYPES
@pytest.mark.parametrize("W", [2, 3, 4])
def test_single_tokens_follow_the_sequence(dtype, W):
    """Token by token from a prompt's state, some slots resting: the same bits as the sequence."""
    from paper_2608_15533_amd import deltalog as D
    lens = [9, 5, 0, 1]
    x = R.conv_inputs(lens, 136, W, dtype, B=6, seed=4)
    c = L.run("conv", x, backward=False)
    s, y, at = c.x["s"].clone(), torch.full_like(c.y, L.FILL), [0, 9, 14, 14]
    for t in range(9):
        live = [i for i in range(4) if t < lens[i]]
        rows = c.x["x"][[at[i] + t for i in live]].contiguous()
        slots = torch.tensor([x["slots"][i] for i in live], dtype=torch.int32, device="cuda")
        out = torch.empty_like(rows)
        D.dl_conv_step(c.desc, s, s, D.ConvRows(c.desc, len(live), rows, c.x["w"], c.x["bias"]), out,
                       slots=slots)
        y[[at[i] + t for i in live]] = out
    assert torch.equal(y, c.y)
    assert torch.equal(s[x["slots"]], c.s_out[x["slots"]])
    rest = [i for i in range(6) if i not in x["slots"]]
    assert torch.equal(s[rest], c.x["s"][rest])


def test_step_leaves_slots_that_do_not_exist():
    from paper_2608_15533_amd import deltalog as D
    x = L.device(R.conv_inputs([3], 64, 4, F32, B=3, seed=5))
    desc = D.make_conv_desc(3, 64, 4, "f32")
    s, y = torch.full_like(x["s"], L.FILL), torch.full((3, 64), L.FILL, device="cuda")
    D.dl_conv_step(desc, x["s"], s, D.ConvRows(desc, 3, x["x"], x["w"], x["bias"]), y,
                   slots=torch.tensor([2, -1, 3], dtype=torch.int32, device="cuda"))
    assert torch.all(y[1:] == L.FILL) and torch.all(s[:2] == L.FILL)
    assert not torch.any(y[0] == L.FILL) and torch.equal(s[2, :2], x["s"][2, 1:])


def test_in_place_and_again():
    x = R.conv_inputs([70, 1, 0, 33], 264, 4, BF16, seed=6)
    c = L.run("conv", x)
    first = {k: v.clone() for k, v in c.results().items()}
    c.ws.fill_(0xff)
    c.forward()
    c.backward()
    assert all(torch.equal(v, first[k]) for k, v in c.results().items())
    c.s_in = c.x["s"].clone()
    c.forward(c.s_in)
    assert torch.equal(c.s_in, first["s"]) and torch.equal(c.y, first["y"])


def test_infinities_and_not_a_number_reach_their_taps_only():
    x = R.conv_inputs([40, 40], 64, 3, F32, seed=7)
    clean = L.run("conv", x)
    x["x"][10, 3], x["x"][20, 5], x["x"][39, 9] = float("nan"), float("inf"), float("-inf")
    bad = L.run("conv", x)
    touched = torch.zeros(80, 64, dtype=torch.bool)
    for t, c in ((10, 3), (20, 5), (39, 9)):
        touched[t:min(t + 3, 40), c] = True
    same = bad.y.cpu() == clean.y.cpu()
    assert torch.equal(~same, touched)
    around = torch.zeros_like(touched)
    for t, c in ((10, 3), (20, 5), (39, 9)):
        around[max(t - 2, 0):min(t + 3, 40), c] = True
    assert torch.all((bad.grads.dx.cpu() == clean.grads.dx.cpu()) | around)


def test_bad_slots_are_skipped():
    x = R.conv_inputs([20, 30, 40], 64, 4, F32, seed=8)
    x["slots"] = [2, 0, 1]
    want = R.conv_expected(x)
    c = L.Packed("conv", x)
    c.slots[1] = 9
    c.build()
    c.forward()
    c.backward()
    assert c.tables.err.item() == 1
    for got, ref in ((c.y, want["out"][0]), (c.grads.dx, want["grads"]["x"])):
        assert R.rel(got[:20], ref[:20]) <= R.TOL["conv"] and R.rel(got[50:], ref[50:]) <= R.TOL["conv"]
    assert torch.all(c.y[20:50] == L.FILL) and torch.all(c.grads.dx[20:50] == 0)
    assert torch.all(c.s_out[0] == L.FILL)
