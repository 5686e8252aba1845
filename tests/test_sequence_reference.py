"""The sequence tests' 64-bit reference against the oracle's token step and against
differences (CPU)."""

import numpy as np
import pytest
import torch

from oracle import eager as OE
import sequence_reference as R


@pytest.mark.parametrize("op", R.OPS)
def test_scan_is_the_oracles_step_repeated(op):
    x = R.inputs(op, [5, 0, 1, 9], 2, 64, 128, seed=3)
    out = R.expected(op, x)
    at = 0
    for i, n in enumerate(x["lens"]):
        S = x["S"][x["slots"][i]].double().numpy()
        for t in range(at, at + n):
            row = {k: None if x[k] is None else x[k][t].double().numpy()
                   for k in ("q", "k", "v", "lam", "beta")}
            u = None if x["u"] is None else x["u"].double().numpy()
            S, o = OE.eager_step(op, S, row["q"], row["k"], row["v"], row["beta"], row["lam"], u=u)
            np.testing.assert_allclose(out["o"][t].numpy(), o, rtol=1e-12, atol=1e-13)
        np.testing.assert_allclose(out["S"][x["slots"][i]].numpy(), S, rtol=1e-12, atol=1e-13)
        at += n


@pytest.mark.parametrize("op", R.OPS)
def test_gradients_against_differences(op):
    """Central differences with step h along a random direction of every input: off by
    h^2 / 6 of a third derivative of order 1, 1e-8 at h = 1e-4 (in 64 bits rounding adds less)."""
    x = R.inputs(op, [3, 6], 1, 64, 64, seed=5)
    g = R.expected(op, x, grads=True)["grads"]

    def loss(y):
        out = R.expected(op, y)
        return (out["o"] * x["do"].double()).sum() + sum(
            (out["S"][s] * x["dS"][s].double()).sum() for s in x["slots"])

    gen = torch.Generator().manual_seed(1)
    for name, dname in R.GRADS.items():
        if x[name] is None:
            continue
        d = torch.randn(x[name].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        up, dn = dict(x), dict(x)
        up[name], dn[name] = x[name].double() + h * d, x[name].double() - h * d
        slope = (loss(up) - loss(dn)) / (2 * h)
        want = (g[dname] * d).sum()
        assert abs(slope - want) <= 1e-5 * max(1.0, abs(want)), name
