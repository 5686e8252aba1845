"""The operators around a recurrence in 64 bits (torch, CPU), differentiable: short causal
convolution, selective scan, norms of queries and keys.  Not collected by pytest.

Tolerances, relative Frobenius errors unless said otherwise.  A bf16 output is a value rounded once,
by at most half a step: eps / 2 = 2^-8 of itself.  fp32 arithmetic before it, EPS = 2^-24 a rounding:

* convolution: at most 5 products and sums, an exponential of an argument up to 20 (its rounding
  weighs 20 EPS where e^-a matters), a reciprocal: below 64 EPS = 4e-6.
* norms: a sum of 128 squares (each rounding is EPS of a growing sum: below 128 EPS, half of it
  after the root), a root, four products, two turned terms: below 128 EPS = 8e-6.
* scan: a state is a sum over tokens of terms that went through as many products as there are tokens
  behind them; each step rounds three times and its decay is an exponential whose argument, at most
  100 where it matters at all, carries two roundings.  Decays forget: with e^-0.001 a token the
  weight of roundings is a few hundred steps long, 3 * 300 EPS in the worst case, which errors of
  either sign reach the square root of.  Bar: 1024 EPS = 6e-5.  Sums over tokens and channels
  (gradients of parameters, of B and C) add at most EPS of the sum of magnitudes a term; they are
  compared with the magnitudes' sum in the denominator where they cancel (see ``rel``).
"""

import math

import torch

F32, BF16 = torch.float32, torch.bfloat16
EPS = 2.0 ** -24
TOL = {"conv": 64 * EPS, "qk": 128 * EPS, "ssm": 1024 * EPS}


def tol(op, dtype):
    return TOL[op] + (torch.finfo(BF16).eps / 2 if dtype == BF16 else 0.0)


def rel(x, ref):
    x, ref = x.detach().double().cpu(), ref.detach().double().cpu()
    den = ref.norm().item()
    return (x - ref).norm().item() / den if den else x.norm().item()


def _normal(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *shape: torch.randn(shape, generator=g, dtype=torch.float64)


def _rows(x, dtype, spare):
    """Rounded to storage, with ``spare`` rows of NaN behind (they belong to nobody)."""
    x = x.to(dtype)
    return torch.cat([x, torch.full((spare,) + x.shape[1:], math.nan, dtype=dtype)])


def _slots(n, B, seed):
    return torch.randperm(B, generator=torch.Generator().manual_seed(seed + 7))[:n].tolist()


# ------------------------------------------------------------------ convolution
def conv_inputs(lens, D, W, dtype=F32, bias=True, B=None, seed=0, spare=0):
    z, N = _normal(seed), sum(lens)
    B = len(lens) if B is None else B
    return {"x": _rows(z(N, D), dtype, spare), "w": (z(D, W) / 2).to(F32),
            "bias": (0.3 * z(D)).to(F32) if bias else None, "s": z(B, W - 1, D).to(dtype),
            "dy": _rows(z(N, D), dtype, spare), "ds": z(B, W - 1, D).to(dtype),
            "lens": list(lens), "slots": _slots(len(lens), B, seed)}


def conv(v, lens, slots, act):
    W = v["w"].shape[1]
    ys, final, at = [], list(v["s"].unbind(0)), 0
    for i, n in enumerate(lens):
        e = torch.cat([v["s"][slots[i]], v["x"][at:at + n]])
        a = sum(e[j:j + n] * v["w"][:, j] for j in range(W))
        if v["bias"] is not None:
            a = a + v["bias"]
        ys.append(a * torch.sigmoid(a) if act == "silu" else a)
        final[slots[i]] = e[n:]
        at += n
    return torch.cat(ys), torch.stack(final)


# ------------------------------------------------------------------ selective scan
def ssm_inputs(lens, D, S, dtype=F32, gate=True, skip=True, bias=True, B=None, seed=0, spare=0,
               step=0.0):
    """``step`` is added to the steps before the softplus: 0 forgets within a few tokens, -5 keeps
    hundreds."""
    z, N = _normal(seed), sum(lens)
    B = len(lens) if B is None else B
    return {"x": _rows(z(N, D), dtype, spare), "dt": _rows(z(N, D) + step, dtype, spare),
            "A": -(torch.arange(1, S + 1) * torch.exp(0.2 * z(D, S))).to(F32),
            "B": _rows(z(N, S), dtype, spare), "C": _rows(z(N, S), dtype, spare),
            "skip": (1 + 0.3 * z(D)).to(F32) if skip else None,
            "bias": (0.3 * z(D)).to(F32) if bias else None,
            "z": _rows(z(N, D), dtype, spare) if gate else None, "s": z(B, D, S).to(F32),
            "dy": _rows(z(N, D), dtype, spare), "ds": z(B, D, S).to(F32),
            "lens": list(lens), "slots": _slots(len(lens), B, seed)}


def ssm(v, lens, slots, act=None):
    raw = v["dt"] if v["bias"] is None else v["dt"] + v["bias"]
    delta = torch.nn.functional.softplus(raw, threshold=1e9)
    ys, final, at = [], list(v["s"].unbind(0)), 0
    for i, n in enumerate(lens):
        h = v["s"][slots[i]]
        for t in range(at, at + n):
            h = torch.exp(delta[t][:, None] * v["A"]) * h + (delta[t] * v["x"][t])[:, None] * v["B"][t]
            ys.append((h * v["C"][t]).sum(-1))
        final[slots[i]] = h
        at += n
    y = torch.stack(ys) if ys else torch.zeros_like(v["x"])
    if v["skip"] is not None:
        y = y + v["skip"] * v["x"]
    if v["z"] is not None:
        y = y * v["z"] * torch.sigmoid(v["z"])
    return y, torch.stack(final)


# ------------------------------------------------------------------ queries and keys
def qk_inputs(n, H, d, rot, rep=1, dtype=F32, weight=True, far=5000, seed=0):
    z = _normal(seed)
    g = torch.Generator().manual_seed(seed + 1)
    w = lambda: (1 + 0.3 * z(d)).to(F32) if weight else None  # noqa: E731
    return {"q": z(n, H, d).to(dtype), "k": z(n, H, d).to(dtype), "wq": w(), "wk": w(),
            "pos": torch.randint(0, far, (n,), generator=g, dtype=torch.int32),
            "freq": (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))).to(F32),
            "dqo": z(n, H * rep, d).to(dtype), "dko": z(n, H * rep, d).to(dtype)}


def qk(v, norm, turn, rot, rep, q_scale, eps=1e-6):
    angle = v["pos"].double()[:, None] * v["freq"].double()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    out = []
    for name, scale in (("q", q_scale), ("k", 1.0)):
        y = v[name]
        if norm != "none":
            y = y * (y.square().sum(-1, keepdim=True) / (y.shape[-1] if norm == "rms" else 1) + eps) ** -0.5
        if v["w" + name] is not None:
            y = y * v["w" + name]
        y = y * scale
        if turn != "none":
            first, second = (y[..., :rot // 2], y[..., rot // 2:rot]) if turn == "halves" else (
                y[..., 0:rot:2], y[..., 1:rot:2])
            a, b = first * cos - second * sin, first * sin + second * cos
            y = torch.cat([torch.cat([a, b], -1) if turn == "halves" else torch.stack([a, b], -1).flatten(-2),
                           y[..., rot:]], -1)
        out.append(y.repeat_interleave(rep, -2))
    return tuple(out)


# ------------------------------------------------------------------ outputs and gradients
def expected(f, x, leaves, ends, grads=True, zero_start=False, final_grad=True):
    """Outputs of ``f`` (a function of the 64-bit leaves) over the rows in use, and the gradients of
    (outputs . ends): a dict of 64-bit tensors."""
    N = sum(x["lens"]) if "lens" in x else None
    v = dict(x)
    for k in leaves:
        if x[k] is None:
            continue
        t = x[k].double() if N is None or k in ("w", "bias", "A", "skip", "s") else x[k][:N].double()
        t = torch.zeros_like(t) if k == "s" and zero_start else t.clone()
        v[k] = t.requires_grad_(grads)
    outs = f(v)
    res = {"out": [o.detach() for o in outs], "grads": {}}
    if grads:
        loss = 0.0
        for o, e in zip(outs, ends):
            if N is not None and e == "ds":
                if final_grad:
                    for s in x["slots"]:
                        loss = loss + (o[s] * x[e][s].double()).sum()
            else:
                loss = loss + (o * x[e][:o.shape[0]].double()).sum()
        names = [k for k in leaves if x[k] is not None]
        got = torch.autograd.grad(loss, [v[k] for k in names], allow_unused=True)
        res["grads"] = {k: torch.zeros_like(v[k]) if g is None else g for k, g in zip(names, got)}
    return res


def conv_expected(x, act="silu", **kw):
    return expected(lambda v: conv(v, x["lens"], x["slots"], act), x, ("x", "w", "bias", "s"),
                    ("dy", "ds"), **kw)


def ssm_expected(x, **kw):
    return expected(lambda v: ssm(v, x["lens"], x["slots"]), x,
                    ("x", "dt", "A", "B", "C", "skip", "bias", "z", "s"), ("dy", "ds"), **kw)


def qk_expected(x, norm, turn, rot, rep, q_scale, **kw):
    return expected(lambda v: qk(v, norm, turn, rot, rep, q_scale), x, ("q", "k", "wq", "wk"),
                    ("dqo", "dko"), **kw)
