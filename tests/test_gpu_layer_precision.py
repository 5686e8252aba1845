"""The softplus of steps and the sigmoids around a recurrence, value by value against 64 bits, over arguments
from where e^-|x| is just a normal fp32 number.

Bars in EPS = 2^-24, a rounding of fp32; the hardware's exponential and reciprocal are good to a unit in the last
place, 2 EPS.  e^-a = 2^t e^d with t = -a log2 e as rounded and d = -a - t ln 2: 2 for 2^t, 1 for the sum with 2^t d,
a / 16 (0.05 a) for ln 2 as an fp32 number.

* softplus, x < 0: 2 artanh(q), q = e / (2 + e): 3 + a / 16 for e, 1 for 2 + e, 2 for its reciprocal, 1 for the
  product, 1.3 for the series: 9 + a / 16.  x > 0: the same of a part, and one more rounding: 10 + a / 16.
* sigmoid: 2 + a / 16 for e, 1 for 1 + e, 2 for its reciprocal, 1 for the sum with its correction: 6 + a / 16; times x or
  another rounded product: 8 + a / 16."""

import pytest
import torch

import layer_reference as R

pytestmark = pytest.mark.gpu

F32, F64, EPS = torch.float32, torch.float64, R.EPS
N = 4096


def spread(lo, hi):
    """N numbers over the range, none of them round."""
    return torch.linspace(lo, hi, N, dtype=F64).add(0.37 * (hi - lo) / N * torch.sin(torch.arange(N))).to(F32)


def worst(got, want, bar):
    """The largest error in units of its bar."""
    off = (got.double().cpu() - want).abs()
    return (off / (bar * EPS).clamp(min=1e-300)).max().item()


class Scan:
    """One token of N channels whose state is its input alone: y = (softplus(dt) + skip) silu(z)."""

    def __init__(self, dt, z=None, skip=None):
        from paper_2608_15533_amd import deltalog as D
        self.D = D
        one = torch.zeros(1, 16, device="cuda")
        one[0, 5] = 1.0
        self.desc = D.make_ssm_desc(1, N, 16, "f32")
        self.rows = D.SsmRows(self.desc, 1, torch.ones(1, N, device="cuda"), dt.cuda()[None],
                              -torch.ones(N, 16, device="cuda"), one, one, z=None if z is None else z.cuda()[None],
                              skip=None if skip is None else torch.full((N,), skip, device="cuda"))
        self.y, self.h = torch.empty(1, N, device="cuda"), torch.zeros(1, N, 16, device="cuda")

    def step(self):
        self.D.dl_ssm_step(self.desc, self.h, torch.empty_like(self.h), self.rows, self.y)
        return self.y[0]

    def prefill(self, backward=False):
        D = self.D
        tables = D.ChunkTables(1, 1)
        D.dl_chunk_tables(torch.ones(1, dtype=torch.int32, device="cuda"), tables)
        ws = D.ssm_workspace(self.desc, 1, 1, backward=True)
        D.dl_ssm_prefill(self.desc, self.h, torch.empty_like(self.h), self.rows, self.y, tables, ws)
        if not backward:
            return self.y[0]
        g = D.SsmGrads(self.desc, self.rows)
        D.dl_ssm_backward(self.desc, self.h, self.rows, torch.ones_like(self.y), None, g, tables, ws)
        return g


@pytest.mark.parametrize("form", ["step", "prefill"])
@pytest.mark.parametrize("lo,hi", [(-87.0, -20.0), (-20.0, 0.0), (0.0, 87.0)])
def test_steps_that_barely_move(form, lo, hi):
    x = spread(lo, hi)
    y = getattr(Scan(x), form)()
    a = x.double()
    want = a.clamp(min=0) + torch.log1p(torch.exp(-a.abs()))
    assert worst(y, want, (10 + a.abs() / 16) * want) <= 1


@pytest.mark.parametrize("lo,hi", [(-86.0, -20.0), (-20.0, 0.0), (0.0, 86.0)])
def test_gradients_of_steps_that_barely_move(lo, hi):
    x = spread(lo, hi)
    g = Scan(x).prefill(backward=True)
    want = torch.sigmoid(x.double())
    assert worst(g.ddt[0], want, (8 + x.double().abs() / 16) * want) <= 1


def slope(z):
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s)), s * (1 + z.abs() * (1 - s))   # and its terms' magnitudes


@pytest.mark.parametrize("lo,hi", [(-85.0, -20.0), (-20.0, 0.0), (0.0, 85.0)])
def test_gates(lo, hi):
    """Of the scan, its step and its gradients: skip 2 and a step near zero, so that y before the gate is 2.
    The slope s (1 + z (1 - s)): s twice, four more roundings, of the terms' magnitudes: 20 + a / 8."""
    z = spread(lo, hi)
    c = Scan(torch.full((N,), -87.0), z, 2.0)
    a = z.double()
    want, bar = 2 * a * torch.sigmoid(a), 8 + a.abs() / 16
    assert worst(c.step().clone(), want, bar * want.abs()) <= 1
    assert worst(c.prefill().clone(), want, bar * want.abs()) <= 1
    d, size = slope(a)
    g = c.prefill(backward=True)
    assert worst(g.dz[0], 2 * d, (20 + a.abs() / 8) * 2 * size) <= 1
    assert worst(g.dx[0], want, (bar + 1) * want.abs()) <= 1


@pytest.mark.parametrize("lo,hi", [(-85.0, -20.0), (-20.0, 0.0), (0.0, 85.0)])
def test_activations_of_the_convolution(lo, hi):
    """The newest input alone: y = silu(x), its gradient the slope."""
    from paper_2608_15533_amd import deltalog as D
    x = spread(lo, hi)
    a = x.double()
    desc = D.make_conv_desc(1, N, 2, "f32")
    w = torch.zeros(N, 2, device="cuda")
    w[:, 1] = 1.0
    rows = D.ConvRows(desc, 1, x.cuda()[None], w)
    s, y = torch.zeros(1, 1, N, device="cuda"), torch.empty(1, N, device="cuda")
    want, bar = a * torch.sigmoid(a), (8 + a.abs() / 16)
    D.dl_conv_step(desc, s, torch.empty_like(s), rows, y)
    assert worst(y[0], want, bar * want.abs()) <= 1
    tables = D.ChunkTables(1, 1)
    D.dl_chunk_tables(torch.ones(1, dtype=torch.int32, device="cuda"), tables)
    D.dl_conv_prefill(desc, s, torch.empty_like(s), rows, y.zero_(), tables)
    assert worst(y[0], want, bar * want.abs()) <= 1
    g = D.ConvGrads(desc, rows)
    D.dl_conv_backward(desc, s, rows, torch.ones_like(y), None, g, tables, D.conv_workspace(desc, 1, 1))
    d, size = slope(a)
    assert worst(g.dx[0], d, (20 + a.abs() / 8) * size) <= 1


def test_ends_of_the_range():
    """A step of -inf does nothing and has no gradient (a token that is masked that way), one of +inf is not finite
    (nor is its product with a B of 0); a gate of +inf is open, as by the definition."""
    inf, nan = float("inf"), float("nan")
    x = torch.full((N,), 0.5)
    x[0], x[1], x[2], x[3], x[4], x[5] = -inf, -200.0, inf, nan, 1e30, -3e38
    for y in (Scan(x).step(), Scan(x).prefill()):
        y = y.cpu()
        assert y[0] == 0 and y[1] == 0 and y[5] == 0 and y[4] == x[4] and not torch.isfinite(y[2]) and torch.isnan(y[3])
    g = Scan(x).prefill(backward=True).ddt[0].cpu()
    assert g[0] == 0 and g[1] == 0 and g[5] == 0 and g[4] == 1 and torch.isnan(g[3])
    z = torch.full((N,), 0.5)
    z[0], z[1], z[2], z[3], z[4] = -200.0, 200.0, inf, nan, -1e30
    c = Scan(torch.full((N,), -87.0), z, 2.0)
    for y in (c.step().clone(), c.prefill().clone()):
        y = y.cpu()
        assert y[0] == 0 and y[1] == 400 and y[2] == inf and torch.isnan(y[3]) and y[4] == 0


@pytest.mark.parametrize("norm", ["l2", "rms"])
def test_zero_heads_under_the_smallest_eps(norm):
    """eps = 2^-126: heads of zeros are zero, their gradient is the upper one times eps^-1/2."""
    from paper_2608_15533_amd import deltalog as D
    eps = 2.0 ** -126
    desc = D.make_qk_desc(3, 64, norm, in_dtype="f32", eps=eps)
    q = torch.zeros(5, 3, 64, device="cuda")
    rows = D.QkRows(desc, 5, q, q)
    out = [torch.full_like(q, 7.0) for _ in range(2)]
    D.dl_qk_norm(desc, rows, *out)
    assert not any(torch.any(o) for o in out)
    g, up = D.QkGrads(desc, rows), torch.full_like(q, 2.0 ** -70)
    D.dl_qk_norm_backward(desc, rows, up, up, g, D.qk_workspace(desc, 5))
    for d in (g.dq, g.dk):
        assert torch.all((d * 2.0 ** 7 - 1).abs() <= 4 * EPS)     # 2^63 to a unit in the last place


def test_heads_beyond_fp32_come_out_0():
    """Values whose squares overflow have the norm infinity; the other heads are as without them."""
    from paper_2608_15533_amd import deltalog as D
    desc = D.make_qk_desc(2, 64, "rms", in_dtype="f32")
    q = torch.ones(3, 2, 64, device="cuda")
    q[1, 0] = 1e25
    rows = D.QkRows(desc, 3, q, q)
    out = [torch.full_like(q, 7.0) for _ in range(2)]
    D.dl_qk_norm(desc, rows, *out)
    g, up = D.QkGrads(desc, rows), torch.ones_like(q)
    D.dl_qk_norm_backward(desc, rows, up, up, g, D.qk_workspace(desc, 3))
    for o, d in zip(out, (g.dq, g.dk)):
        assert not torch.any(o[1, 0]) and not torch.any(d[1, 0])
        o[1, 0] = 1
        assert torch.all((o - 1).abs() <= 16 * EPS + 1e-6)          # (1 + eps)^-1/2
