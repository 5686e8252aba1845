"""Whole-sequence recurrence in 64 bits, token by token, differentiable (torch, CPU).  Not
collected by pytest.  Shapes: q, k [N,H,dk], v [N,H,dv], lam [N,H] | [N,H,dk] | None, beta [N,H]
| None, u [H,dk] | None, S [B,H,dk,dv]; sequences packed one after the other."""

import math

import torch

OPS = ("gdn", "kda", "rwkv6", "linattn", "retnet", "gla")
DELTA = ("gdn", "kda")
PER_KEY = ("kda", "rwkv6", "gla")

# Relative Frobenius error of fp32 outputs.  An fp32 operand goes to the matrix cores as two
# bf16 numbers: off by 2^-18 of itself, and one more 2^-18 of a product for the term left out.
# An output comes through at most five products in a row (gradients of k: pairs, E, states, Z,
# keys), each with two split operands: 5 * 3 * 2^-18 = 5.7e-5 if every error had the same sign;
# fp32 sums and exponentials add a few 2^-24 per term.  The library's bar for fp32 is 1e-4.
TOL_F32 = 1e-4
# A bf16 output is that rounded once, by at most half a step.
TOL_BF16 = TOL_F32 + torch.finfo(torch.bfloat16).eps / 2


def tol(dtype):
    return TOL_BF16 if dtype == torch.bfloat16 else TOL_F32


def scan(op, lens, slots, q, k, v, lam, beta, u, S):
    """(o [N,H,dv], final states [B,H,dk,dv]); float64 in, float64 out."""
    o, final, at = [], list(S.unbind(0)), 0
    for i, n in enumerate(lens):
        s = S[slots[i]]
        for t in range(at, at + n):
            before = s
            if lam is not None:
                s = s * torch.exp(lam[t] if lam.dim() == 3 else lam[t][:, None])[..., None]
            b = v[t]
            if op in DELTA:
                b = beta[t][:, None] * (v[t] - (k[t][..., None] * s).sum(-2))
            s = s + k[t][..., None] * b[:, None, :]
            if op == "rwkv6":
                read = before + (u * k[t])[..., None] * v[t][:, None, :]
            else:
                read = s
            o.append((q[t][..., None] * read).sum(-2))
        final[slots[i]] = s
        at += n
    out = torch.stack(o) if o else torch.zeros((0,) + v.shape[1:], dtype=v.dtype)
    return out, torch.stack(final)


def inputs(op, lens, H, dk, dv, dtype=torch.float32, state=torch.float32, B=None, seed=0,
           spare=0, decay=1.0):
    """Seeded CPU tensors in their storage types: a dict with q, k, v, lam, beta, u, S, lens,
    slots, do, dS.  ``spare`` more token rows behind the last sequence hold NaN (they belong to
    nobody); ``decay`` scales the log-decays."""
    g = torch.Generator().manual_seed(seed)
    N, n = sum(lens), len(lens)
    B = n if B is None else B

    def z(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float64)

    def rows(x, t):
        x = x.to(t)
        return x if not spare else torch.cat([x, torch.full((spare,) + x.shape[1:], math.nan,
                                                            dtype=t)])

    q, k = z(N, H, dk), z(N, H, dk)
    if op == "linattn":
        q, k = torch.nn.functional.elu(q) + 1, torch.nn.functional.elu(k) + 1
    if op != "rwkv6":
        q, k = q / q.norm(dim=-1, keepdim=True), k / k.norm(dim=-1, keepdim=True)
    gate = z(N, H, dk) if op in PER_KEY else z(N, H)
    lam = {"gdn": torch.nn.functional.logsigmoid(3 + 0.5 * gate),
           "kda": -torch.nn.functional.softplus(gate) / 16,
           "rwkv6": -torch.exp(-0.5 + 0.5 * gate), "linattn": None,
           "retnet": torch.log1p(-(2.0 ** (-5 - 5 * torch.arange(H) / H))).expand(N, H),
           "gla": torch.nn.functional.logsigmoid(gate) / 16}[op]
    f32 = torch.float32
    return {
        "q": rows(q, dtype), "k": rows(k, dtype), "v": rows(z(N, H, dv), dtype),
        "lam": None if lam is None else rows(decay * lam, f32),
        "beta": rows(torch.sigmoid(z(N, H)), f32) if op in DELTA else None,
        "u": (0.1 * z(H, dk)).to(f32) if op == "rwkv6" else None,
        "S": (0.1 * z(B, H, dk, dv)).to(state), "do": rows(z(N, H, dv), dtype),
        "dS": (0.1 * z(B, H, dk, dv)).to(state), "lens": list(lens),
        "slots": torch.randperm(B, generator=g)[:n].tolist(),
    }


GRADS = {"q": "dq", "k": "dk", "v": "dv", "lam": "dlam", "beta": "dbeta", "u": "du", "S": "dS"}


def expected(op, x, grads=False, zero_start=False, dS=True):
    """What dl_prefill (and dl_prefill_backward) compute for ``inputs``: o, S and, with
    ``grads``, dq, dk, dv, dlam, dbeta, du, dS, in 64 bits over the rows in use."""
    N = sum(x["lens"])
    y = {}
    for name in GRADS:
        t = x[name]
        if t is not None:
            t = (t if name in ("u", "S") else t[:N]).double()
            t = torch.zeros_like(t) if name == "S" and zero_start else t.clone()
            t.requires_grad_(grads)
        y[name] = t
    o, S = scan(op, x["lens"], x["slots"], y["q"], y["k"], y["v"], y["lam"], y["beta"], y["u"],
                y["S"])
    out = {"o": o.detach(), "S": S.detach()}
    if grads:
        loss = (o * x["do"][:N].double()).sum()
        if dS:
            for s in x["slots"]:
                loss = loss + (S[s] * x["dS"][s].double()).sum()
        names = [n for n in GRADS if y[n] is not None]
        got = torch.autograd.grad(loss, [y[n] for n in names], allow_unused=True)
        out["grads"] = {GRADS[n]: torch.zeros_like(y[n]) if d is None else d
                        for n, d in zip(names, got)}
    return out


def rel(x, ref):
    x, ref = x.double().cpu(), ref.double().cpu()
    den = ref.norm().item()
    return (x - ref).norm().item() / den if den else x.norm().item()
