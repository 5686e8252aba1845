"""Differentiable whole-sequence recurrence: ``dl_prefill`` and ``dl_prefill_backward`` as one
torch.autograd function, for training a layer's projections through it."""

import torch
from torch.autograd.function import once_differentiable

from . import deltalog as D


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, tables, q, k, v, lam, beta, u, S0):
        tok = D.Token(desc, tables.tokens, q, k, v, lam, beta, u)
        o = torch.zeros_like(v)
        S = torch.empty((desc.num_slots, desc.heads, desc.dk, desc.dv),
                        dtype=D.state_torch_dtype(desc), device=v.device)
        ws = D.prefill_workspace(desc, tables.n, tables.tokens, device=v.device)
        D.dl_prefill(desc, S0, S, tok, o, tables, ws)
        ctx.desc, ctx.tables = desc, tables
        ctx.save_for_backward(q, k, v, lam, beta, u, S0)
        return o, S

    @staticmethod
    @once_differentiable
    def backward(ctx, d_o, dS):
        q, k, v, lam, beta, u, S0 = ctx.saved_tensors
        desc, tables = ctx.desc, ctx.tables
        tok = D.Token(desc, tables.tokens, q, k, v, lam, beta, u)
        d_o = torch.zeros_like(v) if d_o is None else d_o.contiguous()
        dS = None if dS is None else dS.contiguous()
        grads = D.Grads(desc, tok, S0)
        ws = D.prefill_workspace(desc, tables.n, tables.tokens, backward=True, device=v.device)
        D.dl_prefill_backward(desc, S0, tok, d_o, dS, grads, tables, ws)
        return (None, None, grads.dq, grads.dk, grads.dv, grads.dlam, grads.dbeta, grads.du,
                grads.dS)


def delta_scan(op, q, k, v, lam=None, beta=None, u=None, S0=None, lens=None, state_dtype="f32"):
    """The recurrence ``op`` (a key of ``deltalog.OP_IDS``) over packed sequences.

    q, k [N,H,dk], v [N,H,dv] in bf16 or fp32; lam [N,H] or [N,H,dk], beta [N,H], u [H,dk] as
    the operator needs them (fp32); lens [n] int32 on the device (None: one sequence of N
    tokens); S0 [n,H,dk,dv] initial states in ``state_dtype`` (None: zero).  Returns (o
    [N,H,dv], final states [n,H,dk,dv]); o and every gradient are 0 in rows behind the last
    sequence; lengths that run past the N rows are cut there.  All tensors contiguous.  Gradients once; the states are computed again for
    them, so a call keeps its inputs and nothing else."""
    N, H, dk = q.shape
    if lens is None:
        lens = torch.full((1,), N, dtype=torch.int32, device=q.device)
    n = lens.numel()
    in_dtype = {torch.bfloat16: "bf16", torch.float32: "f32"}.get(q.dtype)
    if in_dtype is None:
        raise ValueError(f"q: dtype {q.dtype}, expected bf16 or fp32")
    desc = D.make_desc(op, n, H, dk, v.shape[-1], 1, in_dtype, state_dtype)
    tables = D.ChunkTables(n, N, device=q.device)
    D.dl_chunk_tables(lens, tables)
    ids = D.OP_IDS[op]
    return _Scan.apply(desc, tables, q, k, v, None if ids == D.DL_OP_LINATTN else lam,
                       beta if ids in D.DELTA_OP_IDS else None,
                       u if ids == D.DL_OP_RWKV6 else None, S0)
