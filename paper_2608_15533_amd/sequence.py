"""Differentiable whole-sequence operators, for training a layer's projections through them:
``delta_scan`` (``dl_prefill`` and ``dl_prefill_backward`` as one torch.autograd function),
``short_conv``, ``selective_scan`` and ``qk_norm`` likewise.

Tables that are passed in may be filled again once a call has been made, for the next batch: a call's
gradients go by the sequences that it had.  (A call that is made again, as activation checkpointing does, reads
its tables again.)

A training step may be captured into a graph, its forward and backward together.  No graph of an
earlier eager step may still hold the same leaves then: autograd would join the captured stream with
the stream of that step, which ends the capture and may end the process."""

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

def _batch(x, lens):
    """(tables of the packed rows x, their slots, whether the caller built them): ``lens`` [n] int32 on
    the device, None (one sequence of all rows) or tables that the caller has built for these rows already."""
    N = x.shape[0]
    if isinstance(lens, D.ChunkTables):
        return lens, lens.num_slots, True
    if lens is None:
        lens = torch.full((1,), N, dtype=torch.int32, device=x.device)
    tables = D.ChunkTables(lens.numel(), N, device=x.device)
    D.dl_chunk_tables(lens, tables)
    return tables, lens.numel(), False


def _for_backward(ctx, tables, given):
    """The tables a call's gradients go by.  Those that the caller has built (``given``) may be filled
    again, for the next batch, before the gradients are asked for."""
    return tables._kept() if given and any(ctx.needs_input_grad) else tables


def _states(s, given, shape, dtype, device):
    """The buffer of a call's final states.  Tables of the caller's may have slots that no sequence has:
    their states pass through, and so do their gradients."""
    return s.clone() if given and s is not None else torch.zeros(shape, dtype=dtype, device=device)


def _type(x, name):
    in_dtype = {torch.bfloat16: "bf16", torch.float32: "f32"}.get(x.dtype)
    if in_dtype is None:
        raise ValueError(f"{name}: dtype {x.dtype}, expected bf16 or fp32")
    return in_dtype


def _dense(t):
    return None if t is None else t.contiguous()


class _Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, tables, given, x, w, bias, s):
        rows = D.ConvRows(desc, tables.tokens, x, w, bias)
        y = torch.zeros(x.shape, dtype=x.dtype, device=x.device)
        out = _states(s, given, (desc.num_slots, desc.width - 1, desc.channels), x.dtype, x.device)
        D.dl_conv_prefill(desc, s, out, rows, y, tables)
        ctx.desc, ctx.tables, ctx.given = desc, _for_backward(ctx, tables, given), given
        ctx.save_for_backward(x, w, bias, s)
        return y, out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds):
        x, w, bias, s = ctx.saved_tensors
        desc, tables = ctx.desc, ctx.tables
        rows = D.ConvRows(desc, tables.tokens, x, w, bias)
        ds = _dense(ds)
        grads = D.ConvGrads(desc, rows, s, ds if ctx.given else None)
        ws = D.conv_workspace(desc, tables.n, tables.tokens, device=x.device)
        D.dl_conv_backward(desc, s, rows, dy.contiguous(), ds, grads, tables, ws)
        return None, None, None, grads.dx, grads.dw, grads.dbias, grads.ds


def short_conv(x, w, bias=None, s0=None, lens=None, activation="silu"):
    """The short causal convolution of every channel over packed sequences.

    x [N,D] in bf16 or fp32 (columns of a wider tensor will do), w [D,W] and bias [D] in fp32; lens [n]
    int32 on the device (None: one sequence), or ``ChunkTables`` of the batch (states are then by slot, those of
    slots without a sequence pass through); s0 [n,W-1,D] the inputs before each sequence (None: zeros).
    Returns (y [N,D], the last W - 1 inputs [n,W-1,D]); y and its gradients are 0 in rows behind the last
    sequence.  Gradients once; a call keeps its inputs and its tables and nothing else."""
    tables, n, given = _batch(x, lens)
    desc = D.make_conv_desc(n, x.shape[1], w.shape[1], _type(x, "x"), activation)
    return _Conv.apply(desc, tables, given, x, w, bias, s0)


class _Ssm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, tables, given, x, dt, A, Bm, Cm, skip, dt_bias, z, h0):
        rows = D.SsmRows(desc, tables.tokens, x, dt, A, Bm, Cm, skip, dt_bias, z)
        y = torch.zeros(x.shape, dtype=x.dtype, device=x.device)
        h = _states(h0, given, (desc.num_slots, desc.channels, desc.states), torch.float32, x.device)
        ws = D.ssm_workspace(desc, tables.n, tables.tokens, device=x.device)
        D.dl_ssm_prefill(desc, h0, h, rows, y, tables, ws)
        ctx.desc, ctx.tables, ctx.given = desc, _for_backward(ctx, tables, given), given
        ctx.save_for_backward(x, dt, A, Bm, Cm, skip, dt_bias, z, h0)
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        x, dt, A, Bm, Cm, skip, dt_bias, z, h0 = ctx.saved_tensors
        desc, tables = ctx.desc, ctx.tables
        rows = D.SsmRows(desc, tables.tokens, x, dt, A, Bm, Cm, skip, dt_bias, z)
        dh = _dense(dh)
        g = D.SsmGrads(desc, rows, h0, dh if ctx.given else None)
        ws = D.ssm_workspace(desc, tables.n, tables.tokens, backward=True, device=x.device)
        D.dl_ssm_backward(desc, h0, rows, dy.contiguous(), dh, g, tables, ws)
        return (None, None, None, g.dx, g.ddt, g.dA, g.dB, g.dC, g.dskip, g.dbias, g.dz, g.ds)


def selective_scan(x, dt, A, Bm, Cm, skip=None, dt_bias=None, z=None, h0=None, lens=None):
    """The selective state space scan over packed sequences.

    x, dt and z (the gate; None: none) [N,D], Bm and Cm [N,S] in bf16 or fp32 (columns of a wider tensor
    will do); A [D,S], skip [D] and dt_bias [D] in fp32; lens as for ``short_conv``; h0 [n,D,S] fp32
    initial states (None: zeros).  Returns (y [N,D], final states [n,D,S]); y and its gradients are 0 in
    rows behind the last sequence.  Gradients once; a call keeps its inputs and its tables and nothing else."""
    tables, n, given = _batch(x, lens)
    desc = D.make_ssm_desc(n, x.shape[1], A.shape[1], _type(x, "x"))
    return _Ssm.apply(desc, tables, given, x, dt, A, Bm, Cm, skip, dt_bias, z, h0)


class _QkNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, tables, q, k, pos, freq, wq, wk):
        n = q.shape[0]
        rows = D.QkRows(desc, n, q, k, pos, freq, wq, wk, tables)
        shape = (n, desc.heads * desc.rep, desc.head_dim)
        qo, ko = (torch.zeros(shape, dtype=t.dtype, device=t.device) for t in (q, k))
        D.dl_qk_norm(desc, rows, qo, ko)
        ctx.desc, ctx.tables = desc, None if tables is None else _for_backward(ctx, tables, True)
        ctx.save_for_backward(q, k, pos, freq, wq, wk)
        return qo, ko

    @staticmethod
    @once_differentiable
    def backward(ctx, dqo, dko):
        q, k, pos, freq, wq, wk = ctx.saved_tensors
        rows = D.QkRows(ctx.desc, q.shape[0], q, k, pos, freq, wq, wk, ctx.tables)
        g = D.QkGrads(ctx.desc, rows)
        ws = D.qk_workspace(ctx.desc, q.shape[0], device=q.device)
        D.dl_qk_norm_backward(ctx.desc, rows, dqo.contiguous(), dko.contiguous(), g, ws)
        return None, None, g.dq, g.dk, None, None, g.dwq, g.dwk


def qk_norm(q, k, pos=None, freq=None, wq=None, wk=None, norm="l2", turn="none", rep=1, q_scale=1.0,
            eps=1e-6, tables=None):
    """Queries and keys [n,H,d] normalised head by head (``norm`` "l2", "rms" or "none"), weighted by wq
    and wk [d] (fp32), queries scaled by ``q_scale``, the first 2 len(freq) places of every head turned by
    the angles pos freq (``turn`` "halves" or "pairs"; pos [n] int32, freq fp32), every head written
    ``rep`` times.  ``tables``: rows behind its sequences are left out (0).  Gradients once, of q, k, wq and wk;
    freq is a constant, which gets none whatever it requires."""
    rot = 0 if turn == "none" else 2 * freq.numel()
    desc = D.make_qk_desc(q.shape[1], q.shape[2], norm, turn, rot, rep, _type(q, "q"), eps, q_scale)
    return _QkNorm.apply(desc, tables, q, k, pos, freq, wq, wk)
