"""Prompts and training sequences through the recurrent layers: what is measured, and the
operators' plain forms.

The decode path (``cases.py``) advances a state by one token.  The operators here take whole
ragged batches of sequences, token rows packed one sequence after the other:

``tables``   ``dl_chunk_tables``: from the request lengths (device memory), the running
             token and chunk counts, one row (sequence, first token row, tokens, slot) per
             chunk of 32 tokens, and the slot of every token row and sequence.
``prefill``  the tables, then ``dl_prefill``: the gated linear recurrence of one layer over
             all tokens, from each sequence's initial state to its final state, with every
             token's output.
``train``    the same followed by ``dl_prefill_backward``: the gradients of every input and
             of the initial states from those of the outputs and of the final states.

Plain forms: the recurrence in blocks of 16 tokens (Eq. 3 unrolled over a block), sequences
padded to the longest, 32 bits throughout; gradients by differentiating exactly that.
"""

import math
import random

import torch

own = False

DELTA = ("gdn", "kda")
PER_KEY = ("kda", "rwkv6", "gla")
OPS = ("gdn", "kda", "rwkv6", "linattn", "retnet", "gla")
CHUNK = 32          # tokens of a chunk in the tables
BLOCK = 16          # tokens the plain form advances at a time


def _case(name, kind, n, tokens, mix, shape, op="gdn", H=1, dk=64, dv=64, inp="bf16",
          state="f32"):
    c = {"kind": kind, "n": n, "tokens": tokens, "mix": mix, "shape": shape}
    if kind != "tables":
        c.update({"op": op, "H": H, "dk": dk, "dv": dv, "in": inp, "state": state})
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Tables of a handful of requests: the latency of a step's bookkeeping.
        _case("tables_n5", "tables", 5, 300, "ragged", 1),
        # Tables of a large packed batch (evaluation, packed training documents).
        _case("tables_n2000", "tables", 2000, 1000003, "ragged", 2),
        # The smallest prompts: a few tokens through the smallest workload's layer.
        _case("prefill_gdn_short_f32", "prefill", 3, 40, "ragged", 3, "gdn", 2, 64, 64, "f32"),
        # Odd everything: rectangular heads, an odd head count, empty and one-token requests.
        _case("prefill_gla_odd_f32", "prefill", 7, 777, "holes", 4, "gla", 5, 64, 128, "f32"),
        # One long prompt: the only parallelism is heads and value columns.
        _case("prefill_gdn_long", "prefill", 1, 8192, "even", 5, "gdn", 32, 128, 128),
        # An admission batch of the per-key workload's layer.
        _case("prefill_kda_ragged", "prefill", 12, 12345, "ragged", 6, "kda", 32, 128, 128),
        # Many middling prompts into 64 x 64 heads with a bf16 state.
        _case("prefill_rwkv6_ragged", "prefill", 32, 16000, "ragged", 7, "rwkv6", 40, 64, 64,
              state="bf16"),
        # The largest prefill: eight long prompts at the headline layer's shape.
        _case("prefill_gdn_b8", "prefill", 8, 32768, "even", 8, "gdn", 32, 128, 128),
        # A training step's layer at the headline shape, equal sequences.
        _case("train_gdn_b2", "train", 2, 4096, "even", 9, "gdn", 32, 128, 128),
        # Packed documents of unequal lengths, per-key decay.
        _case("train_kda_ragged", "train", 6, 3000, "ragged", 10, "kda", 16, 128, 128),
        # The bonus readout's gradients, 64 x 64 heads.
        _case("train_rwkv6_ragged", "train", 9, 4000, "holes", 11, "rwkv6", 40, 64, 64),
        # A small fp32 step (gradient checks, ablations): rectangular heads, scalar decay.
        _case("train_retnet_f32", "train", 3, 500, "ragged", 12, "retnet", 6, 128, 64, "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "prefill", "prefill", "prefill", "train", "train"])
    mix = rng.choice(["ragged", "ragged", "holes", "even"])
    shape = rng.randrange(100, 1 << 20)
    if kind == "tables":
        n = _log_int(rng, 1, 2000)
        return _case("", kind, n, max(n, _log_int(rng, 64, 1000000)), mix, shape)
    op = rng.choice(OPS)
    dk, dv = rng.choice([(128, 128)] * 3 + [(64, 64)] * 2 + [(64, 128), (128, 64)])
    H = rng.choice([2, 3, 5, 8, 16, 24, 32, 40])
    inp = rng.choice(["bf16"] * 3 + ["f32"])
    state = rng.choice(["f32"] * 3 + ["bf16"])
    n = _log_int(rng, 1, 32)
    tokens = _log_int(rng, 16, 32768 if kind == "prefill" else 4096)
    return _case("", kind, n, max(n, min(tokens, 1048576 // H)), mix, shape, op, H, dk, dv, inp,
                 state)


def _lens(c):
    """Request lengths of a case: they add up to its tokens.  ``holes``: every third request
    is empty or has one token; the last request takes what is left."""
    n, total = c["n"], c["tokens"]
    if c["mix"] == "even":
        return [total // n + (i < total % n) for i in range(n)]
    rng = random.Random(c["shape"])
    w = [math.exp(rng.uniform(0, 2.5)) for _ in range(n)]
    s = sum(w)
    lens = [int(total * x / s) for x in w]
    if c["mix"] == "holes":
        lens = [x if i % 3 != 1 else min(x, i % 2) for i, x in enumerate(lens)]
    lens[n - 1] += total - sum(lens)
    return lens


# ------------------------------------------------------------------ inputs
def _unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def prepare(c, seed):
    """Inputs with the distributions of ``workloads.py``; token rows packed."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    n, N = c["n"], c["tokens"]
    st = {"c": c, "lens": torch.tensor(_lens(c), dtype=torch.int32, device="cuda"),
          "slots": torch.randperm(n, generator=g, device="cuda").to(torch.int32)}
    if c["kind"] != "tables":
        op, H, dk, dv = c["op"], c["H"], c["dk"], c["dv"]
        it = torch.bfloat16 if c["in"] == "bf16" else torch.float32
        stt = torch.bfloat16 if c["state"] == "bf16" else torch.float32

        def z(*shape):
            return torch.randn(shape, generator=g, device="cuda")

        q, k = z(N, H, dk), z(N, H, dk)
        if op == "linattn":
            q, k = torch.nn.functional.elu(q) + 1, torch.nn.functional.elu(k) + 1
        if op != "rwkv6":
            q, k = _unit(q), _unit(k)
        st["q"], st["k"], st["v"] = q.to(it), k.to(it), z(N, H, dv).to(it)
        st["lam"] = {
            "gdn": lambda: torch.nn.functional.logsigmoid(3.0 + 0.5 * z(N, H)),
            "kda": lambda: -torch.nn.functional.softplus(z(N, H, dk)) / 16.0,
            "rwkv6": lambda: -torch.exp(-0.5 + 0.5 * z(N, H, dk)),
            "linattn": lambda: None,
            "retnet": lambda: torch.log1p(-(2.0 ** (-5.0 - 5.0 * torch.arange(H, device="cuda")
                                                    / H))).expand(N, H).contiguous(),
            "gla": lambda: torch.nn.functional.logsigmoid(z(N, H, dk)) / 16.0,
        }[op]()
        st["beta"] = torch.sigmoid(z(N, H)) if op in DELTA else None
        st["u"] = 0.1 * z(H, dk) if op == "rwkv6" else None
        st["S0"] = (0.02 * z(n, H, dk, dv)).to(stt)
        if c["kind"] == "train":
            st["do"] = z(N, H, dv).to(it)
            st["dS"] = (0.1 * z(n, H, dk, dv)).to(stt)
    if own:
        st["own"] = _handle(st)
    return st


def _handle(st):
    """What a user's program keeps: the descriptor, buffers for the results, workspaces."""
    from paper_2608_15533_amd import deltalog as D
    c = st["c"]
    h = {"D": D, "tables": D.ChunkTables(c["n"], c["tokens"])}
    if c["kind"] != "tables":
        desc = D.make_desc(c["op"], c["n"], c["H"], c["dk"], c["dv"], 16, c["in"], c["state"])
        h["desc"] = desc
        h["tok"] = D.Token(desc, c["tokens"], st["q"], st["k"], st["v"], st["lam"], st["beta"],
                           st["u"])
        h["o"] = torch.empty_like(st["v"])
        h["S"] = torch.empty_like(st["S0"])
        h["ws"] = D.prefill_workspace(desc, c["n"], c["tokens"], backward=c["kind"] == "train")
        if c["kind"] == "train":
            h["grads"] = D.Grads(desc, h["tok"], st["S0"])
    return h


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    h, kind = st["own"], st["c"]["kind"]
    D, t = h["D"], h["tables"]
    D.dl_chunk_tables(st["lens"], t, slots=st["slots"])
    if kind == "tables":
        return {"cu_tokens": t.cu_tokens, "cu_chunks": t.cu_chunks, "chunks": t.chunks,
                "row_slot": t.row_slot, "seq_slot": t.seq_slot}
    D.dl_prefill(h["desc"], st["S0"], h["S"], h["tok"], h["o"], t, h["ws"])
    out = {"o": h["o"], "S": h["S"]}
    if kind == "train":
        g = h["grads"]
        D.dl_prefill_backward(h["desc"], st["S0"], h["tok"], st["do"], st["dS"], g, t, h["ws"])
        out.update({"dq": g.dq, "dk": g.dk, "dv": g.dv, "dS0": g.dS})
        out.update({k: v for k, v in (("dlam", g.dlam), ("dbeta", g.dbeta), ("du", g.du))
                    if v is not None})
    return out


# ------------------------------------------------------------------ plain forms
def _plain_tables(st):
    c, lens, slots = st["c"], st["lens"].long(), st["slots"].long()
    n, N = c["n"], c["tokens"]
    rows = N // CHUNK + n
    zero = torch.zeros(1, dtype=torch.long, device=lens.device)
    cu_t = torch.cat([zero, torch.cumsum(lens, 0)])
    cu_c = torch.cat([zero, torch.cumsum((lens + CHUNK - 1) // CHUNK, 0)])

    def owner(cu, size):
        """For each of ``size`` places, the last request that starts at or before it."""
        at = torch.zeros(size + 1, dtype=torch.long, device=cu.device)
        at.index_add_(0, cu[:-1].clamp(max=size), torch.ones_like(cu[:-1]))
        return torch.cumsum(at, 0)[:size] - 1

    i = torch.arange(rows, device=lens.device)
    s = owner(cu_c, rows)
    first = cu_t[s] + CHUNK * (i - cu_c[s])
    count = torch.minimum(cu_t[s + 1] - first, torch.full_like(first, CHUNK))
    chunks = torch.stack([s, first, count, slots[s]], 1)
    empty = torch.tensor([-1, 0, 0, -1], device=lens.device)
    chunks = torch.where((i < cu_c[n])[:, None], chunks, empty)
    r = torch.arange(N, device=lens.device)
    row_slot = torch.where(r < cu_t[n], slots[owner(cu_t, N)], torch.full_like(r, -1))
    return {"cu_tokens": cu_t.int(), "cu_chunks": cu_c.int(), "chunks": chunks.int(),
            "row_slot": row_slot.int(), "seq_slot": slots.int()}


def _plain_scan(c, q, k, v, lam, beta, u, S, idx, live):
    """o [N,H,dv] and the final states of packed rows in 32 bits: blocks of 16 tokens, all
    sequences side by side.  ``idx`` [n,T] is the packed row of each padded place, ``live``
    whether it is one; a place that is none has zero key, value, beta and log-decay, which
    leave the state as it is."""
    op, dk = c["op"], c["dk"]
    n, T = idx.shape
    keep = live[:, :, None, None].float()

    def padded(x):                                   # [N,H,d] -> [n,H,T,d]
        return (x[idx] * keep).transpose(1, 2)

    q, k, v = padded(q), padded(k), padded(v)
    H = q.shape[1]
    if lam is None:
        lam = torch.zeros((n, H, T, 1), device=q.device)
    else:
        lam = padded(lam if lam.dim() == 3 else lam[..., None])
    beta = None if beta is None else padded(beta[..., None])
    eye = torch.eye(BLOCK, device=q.device)
    outs = []
    for t in range(0, T, BLOCK):
        qb, kb, vb, lb = (x[:, :, t:t + BLOCK] for x in (q, k, v, lam))
        cum = torch.cumsum(lb, 2)
        qcum = cum - lb if op == "rwkv6" else cum
        kdec, kinv, qdec = kb * torch.exp(cum), kb * torch.exp(-cum), qb * torch.exp(qcum)
        pair = torch.tril(qdec @ kinv.transpose(2, 3), -1 if op == "rwkv6" else 0)
        if op == "rwkv6":
            pair = pair + eye * (qb * u[None, :, None, :] * kb).sum(-1, keepdim=True)
        if op in DELTA:
            bb = beta[:, :, t:t + BLOCK]
            A = bb * torch.tril(kdec @ kinv.transpose(2, 3), -1)
            A2 = A @ A
            A4 = A2 @ A2
            r = bb * (vb - kdec @ S)                 # (I + A) U = r, A strictly lower
            r = r + (A4 @ A4) @ r
            r = r + A4 @ r
            r = r + A2 @ r
            U = r - A @ r
        else:
            U = vb
        outs.append(qdec @ S + pair @ U)
        end = cum[:, :, -1:]
        S = torch.exp(end).transpose(2, 3) * S + (kb * torch.exp(end - cum)).transpose(2, 3) @ U
    o = torch.cat(outs, 2).transpose(1, 2)           # [n,T,H,dv]
    return o[live], S


def _places(lens):
    """Packed rows of the padded places [n,T], T a whole number of blocks, and which live."""
    lens = lens.long()
    start = torch.cumsum(lens, 0) - lens
    T = max(1, -(-int(lens.max()) // BLOCK)) * BLOCK
    at = torch.arange(T, device=lens.device)
    live = at[None, :] < lens[:, None]
    return torch.where(live, start[:, None] + at[None, :], torch.zeros_like(at)[None, :]), live


def _run_plain(st):
    c = st["c"]
    if c["kind"] == "tables":
        return _plain_tables(st)
    train = c["kind"] == "train"
    idx, live = _places(st["lens"])
    slots = st["slots"].long()
    names = [k for k in ("q", "k", "v", "lam", "beta", "u", "S0") if st[k] is not None]
    x = {k: None for k in ("q", "k", "v", "lam", "beta", "u", "S0")}
    x.update({k: st[k].detach().float().requires_grad_(train) for k in names})
    with torch.set_grad_enabled(train):
        o, S = _plain_scan(c, x["q"], x["k"], x["v"], x["lam"], x["beta"], x["u"],
                           x["S0"][slots], idx, live)
    out = {"o": o.detach().to(st["v"].dtype),
           "S": torch.empty_like(st["S0"]).index_copy_(0, slots, S.detach().to(st["S0"].dtype))}
    if train:
        g = torch.autograd.grad([o, S], [x[k] for k in names],
                                [st["do"].float(), st["dS"].float()[slots]])
        out.update({"d" + k: y.to(st[k].dtype) for k, y in zip(names, g)})
    return out


# ------------------------------------------------------------------ work, 64 bits
def work(c):
    n, N = c["n"], c["tokens"]
    if c["kind"] == "tables":
        return {"bytes": 4 * (3 * n + 2 * (n + 1) + 4 * (N // CHUNK + n) + N), "flops": 2 * n + N}
    H, dk, dv = c["H"], c["dk"], c["dv"]
    e, es = (2 if c["in"] == "bf16" else 4), (2 if c["state"] == "bf16" else 4)
    delta = c["op"] in DELTA
    gate = {"linattn": 0, "gdn": 4, "retnet": 4}.get(c["op"], 4 * dk) + (4 if delta else 0)
    once = 4 * H * dk if c["op"] == "rwkv6" else 0
    state = n * H * dk * dv * es
    fwd = N * H * (2 * dk * e + 2 * dv * e + gate) + 2 * state + once
    flops = N * H * dk * dv * (6 if delta else 4)
    if c["kind"] == "train":
        # q, k, v, dO and the gates read again; dq, dk, dv and the gates' gradients written
        fwd += N * H * (4 * dk * e + 3 * dv * e + 2 * gate) + 3 * state + 2 * once
        flops += N * H * dk * dv * (16 if delta else 10)
    return {"bytes": fwd, "flops": flops}


def exact(c, seed):
    """The recurrence token by token in 64 bits, and its adjoint token by token."""
    if c["kind"] == "tables":
        return None
    st = prepare(c, seed)
    op, n, N, H, dk, dv = c["op"], c["n"], c["tokens"], c["H"], c["dk"], c["dv"]
    lens = _lens(c)
    first = [sum(lens[:i]) for i in range(n)]
    f64 = dict(dtype=torch.float64, device="cuda")
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    w = None if st["lam"] is None else torch.exp(st["lam"].double()).reshape(N, H, -1)
    beta = None if st["beta"] is None else st["beta"].double()[..., None]
    u = None if st["u"] is None else st["u"].double()
    slots = st["slots"].long()
    # longest first, so that the sequences still running at step t are the first m
    order = sorted(range(n), key=lambda i: -lens[i])
    begin = torch.tensor([first[i] for i in order], device="cuda")
    where = slots[torch.tensor(order, device="cuda")]
    S = st["S0"].double()[where].clone()
    running, T = [0] * (max(lens) + 1), max(lens)
    for i in order:
        running[lens[i]] += 1
    for t in range(T - 1, -1, -1):
        running[t] += running[t + 1]                 # running[t + 1]: sequences longer than t

    def old(m, r):                                   # decayed state, correction, pair's value
        Sd = S[:m] if w is None else S[:m] * w[r][..., None]
        if beta is None:
            return Sd, None, v[r]
        res = v[r] - (k[r][..., None] * Sd).sum(-2)
        return Sd, res, beta[r] * res

    def forward(t):
        m = running[t + 1]
        r = begin[:m] + t
        before = S[:m].clone() if op == "rwkv6" else None
        Sd, _, b = old(m, r)
        S[:m] = Sd + k[r][..., None] * b[..., None, :]
        if op == "rwkv6":
            before = before + (u * k[r])[..., None] * v[r][..., None, :]
        return r, (q[r][..., None] * (S[:m] if before is None else before)).sum(-2)

    train, every, kept = c["kind"] == "train", 64, []
    o = torch.zeros((N, H, dv), **f64)
    for t in range(T):
        if train and t % every == 0:
            kept.append(S.clone())
        r, y = forward(t)
        o[r] = y
    back = torch.empty_like(S)
    back[where] = S
    out = {"o": o, "S": back}
    if not train:
        return out
    do, G = st["do"].double(), st["dS"].double()[where].clone()
    dq, dkk, dvv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dw = None if w is None else torch.zeros_like(w)
    db = None if beta is None else torch.zeros_like(beta)
    du = None if u is None else torch.zeros_like(u)
    for seg in range(len(kept) - 1, -1, -1):
        S = kept[seg]
        states = []
        for t in range(seg * every, min(T, (seg + 1) * every)):
            states.append(S[:running[t + 1]].clone())
            forward(t)
        for t in range(min(T, (seg + 1) * every) - 1, seg * every - 1, -1):
            m = running[t + 1]
            r = begin[:m] + t
            S = states.pop()
            Sd, res, b = old(m, r)
            kr, g = k[r], do[r]
            if op == "rwkv6":
                dq[r] = (S * g[..., None, :]).sum(-1)
                own_pair = (g * v[r]).sum(-1, keepdim=True)
                dq[r] += own_pair * u * kr
                dkk[r] += own_pair * u * q[r]
                du += (own_pair * q[r] * kr).sum(0)
                dvv[r] += (q[r] * u * kr).sum(-1, keepdim=True) * g
            else:
                dq[r] = ((Sd + kr[..., None] * b[..., None, :]) * g[..., None, :]).sum(-1)
                G[:m] += q[r][..., None] * g[..., None, :]
            Gm = G[:m].clone()
            gb = (Gm * kr[..., None]).sum(-2)
            dkk[r] += (Gm * b[..., None, :]).sum(-1)
            if beta is None:
                dvv[r] += gb
            else:
                db[r] = (gb * res).sum(-1, keepdim=True)
                gb = beta[r] * gb
                dvv[r] += gb
                dkk[r] -= (Sd * gb[..., None, :]).sum(-1)
                Gm = Gm - kr[..., None] * gb[..., None, :]
            if w is not None:
                dl = (Gm * Sd).sum(-1)               # d/dlam = w d/dw, and Sd = w S
                dw[r] = dl if dw.shape[-1] == dk else dl.sum(-1, keepdim=True)
                Gm = Gm * w[r][..., None]
            if op == "rwkv6":
                Gm = Gm + q[r][..., None] * g[..., None, :]
            G[:m] = Gm
    dS0 = torch.empty_like(G)
    dS0[where] = G
    out.update({"dq": dq, "dk": dkk, "dv": dvv, "dS0": dS0})
    if w is not None:
        out["dlam"] = dw.reshape(st["lam"].shape)
    if db is not None:
        out["dbeta"] = db[..., 0]
    if du is not None:
        out["du"] = du
    return out
