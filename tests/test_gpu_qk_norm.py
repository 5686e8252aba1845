"""Norms of queries and keys for each head, with the rotation by position, against 64 bits."""

import pytest
import torch

import layer_harness as L
import layer_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
GRADS = ("dq", "dk", "dwq", "dwk")


class Call:
    def __init__(self, x, norm, turn, rot, rep=1, q_scale=1.0, strided=False, tables=None, eps=1e-6):
        from paper_2608_15533_amd import deltalog as D
        self.D, self.x = D, L.device(x)
        y = self.x
        self.n, H, d = y["q"].shape
        inp = "bf16" if y["q"].dtype == BF16 else "f32"
        self.desc = D.make_qk_desc(H, d, norm, turn, rot, rep, inp, eps, q_scale)
        put = (lambda t: L.wide(t.reshape(self.n, -1)).unflatten(1, (H, d))) if strided else (lambda t: t)
        self.rows = D.QkRows(self.desc, self.n, put(y["q"]), put(y["k"]), y["pos"], y["freq"], y["wq"],
                             y["wk"], tables)
        self.q, self.k = (torch.full((self.n, H * rep, d), L.FILL, dtype=y["q"].dtype, device="cuda")
                          for _ in range(2))
        self.grads, self.ws = D.QkGrads(self.desc, self.rows), D.qk_workspace(self.desc, self.n)
        self.ws.fill_(0xff)

    def forward(self):
        self.D.dl_qk_norm(self.desc, self.rows, self.q, self.k)

    def backward(self):
        self.D.dl_qk_norm_backward(self.desc, self.rows, self.x["dqo"], self.x["dko"], self.grads, self.ws)

    def results(self):
        return {"q": self.q, "k": self.k, **{k: getattr(self.grads, k) for k in GRADS
                                             if getattr(self.grads, k) is not None}}


def check(c, want, n=None):
    for got, ref in zip((c.q, c.k), want["out"]):
        e = R.rel(got[:n], ref)
        assert e <= R.tol("qk", got.dtype), f"output {e:.2e}"
    for k, ref in want["grads"].items():
        got = getattr(c.grads, "d" + k)
        e = R.rel(got if k[0] == "w" else got[:n], ref)
        assert e <= R.tol("qk", got.dtype), f"d{k} {e:.2e}"


@TYPES
@pytest.mark.parametrize("norm", ["l2", "rms", "none"])
@pytest.mark.parametrize("turn,rot", [("none", 0), ("halves", 16), ("halves", 48), ("halves", 64),
                                      ("pairs", 16), ("pairs", 64)])
@pytest.mark.parametrize("n,H,d,rep", [(1, 1, 64, 1), (5, 3, 64, 2), (37, 33, 128, 1), (3, 5, 128, 3)], ids=str)
def test_rows(dtype, norm, turn, rot, n, H, d, rep):
    x = R.qk_inputs(n, H, d, rot, rep, dtype, weight=norm != "l2", seed=n)
    c = Call(x, norm, turn, rot, rep, 0.3)
    c.forward()
    c.backward()
    check(c, R.qk_expected(x, norm, turn, rot, rep, 0.3))


@TYPES
@pytest.mark.parametrize("turn", ["halves", "pairs"])
def test_whole_heads_of_128_and_rows_of_a_wider_tensor(dtype, turn):
    x = R.qk_inputs(33, 4, 128, 128, 2, dtype, seed=1)
    c = Call(x, "rms", turn, 128, 2, strided=True)
    c.forward()
    c.backward()
    check(c, R.qk_expected(x, "rms", turn, 128, 2, 1.0))


def test_many_tokens_and_far_positions():
    """Several tokens a workgroup; positions from the most negative to the largest.  An angle is the
    position times the 32-bit frequency; 64 bits of the product leave 2^31 2^-53 radians."""
    x = R.qk_inputs(9000, 2, 64, 64, 1, F32, seed=2)
    x["pos"][:6] = torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 1 << 20, 12345678], dtype=torch.int32)
    c = Call(x, "l2", "halves", 64)
    c.forward()
    c.backward()
    check(c, R.qk_expected(x, "l2", "halves", 64, 1, 1.0))


@TYPES
def test_heads_of_zeros_and_of_large_values(dtype):
    x = R.qk_inputs(4, 2, 64, 64, 1, dtype, seed=3)
    x["q"][0, 0] = 0
    x["k"][1] = 0
    x["k"][2] *= 2.0 ** 40
    x["q"][3] *= 2.0 ** -40                             # far below eps
    c = Call(x, "rms", "pairs", 64, eps=1e-5)
    c.forward()
    c.backward()
    want = R.expected(lambda v: R.qk(v, "rms", "pairs", 64, 1, 1.0, 1e-5), x, ("q", "k", "wq", "wk"),
                      ("dqo", "dko"))
    assert torch.all(c.q[0, 0] == 0) and torch.all(c.k[1] == 0)
    for name, got in (("q", c.grads.dq), ("k", c.grads.dk)):
        for t in range(4):                              # row by row: they differ in size by 2^80
            assert R.rel(got[t], want["grads"][name][t]) <= R.tol("qk", dtype), (name, t)
    for i, got in enumerate((c.q, c.k)):
        for t in range(4):
            assert R.rel(got[t], want["out"][i][t]) <= R.tol("qk", dtype)


def test_not_a_number_stays_in_its_head():
    x = R.qk_inputs(3, 3, 128, 128, 2, F32, weight=False, seed=4)
    clean = Call(x, "l2", "halves", 128, 2)
    clean.forward()
    clean.backward()
    x["q"][1, 1, 5], x["k"][2, 0, 7] = float("nan"), float("inf")
    bad = Call(x, "l2", "halves", 128, 2)
    bad.forward()
    bad.backward()
    for name, (t, h) in (("q", (1, 1)), ("k", (2, 0))):
        a, b = clean.results()[name].clone(), bad.results()[name].clone()
        assert torch.isnan(b[t, 2 * h:2 * h + 2]).any()
        a[t, 2 * h:2 * h + 2] = b[t, 2 * h:2 * h + 2] = 0
        assert torch.equal(a, b)
        a, b = clean.results()["d" + name].clone(), bad.results()["d" + name].clone()
        a[t, h] = b[t, h] = 0
        assert torch.equal(a, b)


def test_rows_behind_the_last_sequence():
    """With tables, rows in nobody's sequence are neither read into sums nor written."""
    from paper_2608_15533_amd import deltalog as D
    x = R.qk_inputs(50, 3, 64, 32, 1, BF16, seed=5)
    tables = D.ChunkTables(2, 50)
    D.dl_chunk_tables(torch.tensor([20, 23], dtype=torch.int32, device="cuda"), tables)
    for k in ("q", "k", "dqo", "dko"):
        x[k][43:] = float("nan")
    c = Call(x, "rms", "halves", 32, tables=tables)
    c.forward()
    c.backward()
    cut = {k: v[:43] if v.shape[0] == 50 else v for k, v in x.items()}
    check(c, R.qk_expected(cut, "rms", "halves", 32, 1, 1.0), 43)
    assert torch.all(c.q[43:] == L.FILL) and torch.all(c.k[43:] == L.FILL)
    assert torch.all(c.grads.dq[43:] == 0) and torch.all(c.grads.dk[43:] == 0)


def test_again():
    x = R.qk_inputs(3000, 4, 64, 64, 2, BF16, seed=6)
    c = Call(x, "rms", "halves", 64, 2)
    c.forward()
    c.backward()
    first = {k: v.clone() for k, v in c.results().items()}
    c.ws.fill_(0xff)
    c.forward()
    c.backward()
    assert all(torch.equal(v, first[k]) for k, v in c.results().items())
