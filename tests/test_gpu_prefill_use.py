"""Whole-sequence calls as they are used: tables, a prompt followed by decoding, prompts in
parts, training through autograd, capture and replay, other streams, calls in place."""

import numpy as np
import pytest
import torch

import prefill_harness as P
import sequence_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _D():
    from paper_2608_15533_amd import deltalog
    return deltalog


# ------------------------------------------------------------------ tables
def plain_tables(lens, slots, tokens, num_slots):
    D, bad, at = _D(), 0, 0
    cu_t, cu_c, chunks, row_slot, seq_slot = [0], [0], [], [-1] * tokens, []
    for i, n in enumerate(lens):
        if n < 0:
            n, bad = 0, bad | 4
        if at + n > tokens:
            bad |= 4
        n = min(n, tokens - at)
        s = slots[i] if slots is not None else i
        if not 0 <= s < num_slots:
            s, bad = -1, bad | 1
        seq_slot.append(s)
        for first in range(at, at + n, D.DL_CHUNK):
            chunks.append((i, first, min(D.DL_CHUNK, at + n - first), s))
        row_slot[at:at + n] = [s] * n
        at += n
        cu_t.append(at)
        cu_c.append(len(chunks))
    chunks += [(-1, 0, 0, -1)] * (tokens // D.DL_CHUNK + len(lens) - len(chunks))
    return cu_t, cu_c, chunks, row_slot, seq_slot, bad


def check_tables(lens, slots, tokens, num_slots):
    D = _D()
    t = D.ChunkTables(len(lens), tokens, num_slots)
    i32 = dict(dtype=torch.int32, device="cuda")
    D.dl_chunk_tables(torch.tensor(lens, **i32), t,
                      None if slots is None else torch.tensor(slots, **i32))
    cu_t, cu_c, chunks, row_slot, seq_slot, bad = plain_tables(lens, slots, tokens, num_slots)
    assert t.cu_tokens.tolist() == cu_t
    assert t.cu_chunks.tolist() == cu_c
    assert t.seq_slot.tolist() == seq_slot
    assert t.row_slot.tolist() == row_slot
    assert t.chunks.tolist() == [list(c) for c in chunks]
    assert t.err.item() == bad
    count = [cu_c[i + 1] - cu_c[i] for i in range(len(lens))]
    want = list(range(len(lens)))
    if len(lens) <= 1024:
        want.sort(key=lambda i: -count[i])
    assert t.order.tolist() == want


@pytest.mark.parametrize("lens,spare", [
    ([1], 0), ([0], 0), ([0], 5), ([32], 0), ([33, 0, 31], 3), ([0, 0, 7, 0, 64, 0], 1),
    (list(range(40)), 0)], ids=str)
def test_tables(lens, spare):
    check_tables(lens, None, sum(lens) + spare, len(lens))
    check_tables(lens, list(range(len(lens)))[::-1], sum(lens) + spare, len(lens) + 2)


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2049, 4096, 4097, 5000])
def test_tables_of_many_sequences(n):
    g = np.random.default_rng(n)
    lens = g.integers(0, 70, n).tolist()
    check_tables(lens, g.permutation(n).tolist(), sum(lens) + 11, n)


def test_tables_report_what_is_wrong():
    check_tables([5, -3, 9], [0, 1, 2], 20, 3)            # a negative length
    check_tables([5, 30, 9], [0, 1, 2], 20, 3)            # past the rows
    check_tables([5, 3, 9], [0, 7, -1], 20, 3)            # slots outside
    check_tables([2 ** 31 - 1, 2 ** 31 - 1, 4], [0, 1, 2], 20, 3)


def test_bad_slots_and_lengths_touch_nothing_else():
    """A sequence with a bad slot is skipped; one that is cut short ends with the rows."""
    x = R.inputs("gdn", [20, 30, 40], 2, 64, 64, seed=3, B=3)
    x["slots"] = [2, 0, 1]
    want = R.expected("gdn", x, grads=True)
    c = P.Call("gdn", x, backward=True)
    c.slots[1] = 9
    c.build()
    c.forward()
    c.backward()
    assert c.tables.err.item() == 1
    assert R.rel(c.o[:20], want["o"][:20]) <= R.TOL_F32 and R.rel(c.o[50:], want["o"][50:]) <= R.TOL_F32
    assert torch.all(c.o[20:50] == 7.0) and torch.all(c.S_out[0] == 7.0)
    for name in ("dq", "dk", "dv", "dlam", "dbeta"):
        got = getattr(c.grads, name)
        assert torch.all(got[20:50] == 0), name
        assert R.rel(got[:20], want["grads"][name][:20]) <= R.TOL_F32, name


def test_tables_for_more_slots_than_the_state_has():
    """Slots are checked again against the state's own count."""
    x = R.inputs("gla", [20, 30], 2, 64, 64, seed=3)
    c = P.Call("gla", x)
    c.tables = c.D.ChunkTables(2, 50, num_slots=100)
    c.slots[0] = 50
    c.build()
    assert c.tables.err.item() == 0
    c.forward()
    assert torch.all(c.o[:20] == 7.0)
    assert torch.isfinite(c.o).all()


# ------------------------------------------------------------------ a run of calls
@pytest.mark.parametrize("op", R.OPS)
def test_prompt_then_decode(op):
    """Engine: prompts, then decode steps with merges on the way, then one prompt's second part
    and more steps, against the 64-bit recurrence over everything."""
    from paper_2608_15533_amd import decode
    D = _D()
    H, dk, dv, M, layers, lens, steps, more = 2, 64, 128, 3, 2, [37, 0, 5], 5, 33
    desc = D.make_desc(op, 4, H, dk, dv, M, "f32")
    eng = decode.DecodeEngine(desc, layers)
    total = sum(lens)
    x = [R.inputs(op, [total + 3 * 2 * steps + more], H, dk, dv, seed=20 + i)
         for i in range(layers)]
    if op == "rwkv6":
        for i in range(layers):
            eng.inputs[i].u.copy_(x[i]["u"])

    def rows(i, idx):
        return [None if x[i][n] is None else x[i][n][idx].cuda().contiguous()
                for n in ("q", "k", "v", "lam", "beta")]

    slots, outs = eng.prefill(lens, [rows(i, slice(0, total)) for i in range(layers)])
    assert len(slots) == 3 and eng.sched.free_slots == 1
    ran = [[list(range(sum(lens[:j]), sum(lens[:j + 1]))) for j in range(3)] for _ in range(layers)]
    got = [[[outs[i][r].cpu() for r in ran[i][j]] for j in range(3)] for i in range(layers)]
    at = total

    def decode_steps():
        nonlocal at
        for _ in range(steps):
            plan = eng.schedule()
            for j, s in enumerate(slots):
                for i in range(layers):
                    eng.inputs[i].write([plan.row_of(s)], *rows(i, slice(at + j, at + j + 1)))
                    ran[i][j].append(at + j)
            eng.step()
            for j, s in enumerate(slots):
                for i in range(layers):
                    got[i][j].append(eng.output(i, s, plan).cpu().clone())
            at += 3

    decode_steps()
    again, outs = eng.prefill([more], [rows(i, slice(at, at + more)) for i in range(layers)],
                              slots=[slots[0]])
    assert again == [slots[0]]
    for i in range(layers):
        ran[i][0] += list(range(at, at + more))
        got[i][0] += list(outs[i].cpu())
    at += more
    decode_steps()
    assert eng.error_words() == [0] * layers
    for i in range(layers):
        for j, s in enumerate(slots):
            idx = ran[i][j]
            y = {n: None if x[i][n] is None else x[i][n][idx] for n in ("q", "k", "v", "lam", "beta")}
            y.update(u=x[i]["u"], S=torch.zeros(1, H, dk, dv), lens=[len(idx)], slots=[0],
                     do=None, dS=None)
            want = R.expected(op, y)
            assert R.rel(torch.stack(got[i][j]), want["o"]) <= R.TOL_F32
            assert R.rel(eng.flush(s)[i], want["S"][0]) <= R.TOL_F32


def test_engine_refuses():
    from paper_2608_15533_amd import decode
    D = _D()
    desc = D.make_desc("linattn", 2, 2, 64, 64, 4, "f32")
    eng = decode.DecodeEngine(desc, 1)
    z = torch.zeros((6, 2, 64), device="cuda")
    tok = [(z, z, z, None, None)]
    with pytest.raises(decode.SlotError):
        eng.prefill([2, 2, 2], tok)
    with pytest.raises(ValueError):
        eng.prefill([2, 3], tok)                          # rows that do not add up
    with pytest.raises(ValueError):
        eng.prefill([7, -1], tok)
    with pytest.raises(ValueError):
        eng.prefill([6], tok * 2)
    assert eng.sched.free_slots == 2
    slots, _ = eng.prefill([3, 3], tok)
    with pytest.raises(decode.SlotError):
        eng.prefill([6], tok, slots=[5])
    with pytest.raises(ValueError):
        eng.prefill([3, 3], tok, slots=[slots[0]] * 2)
    assert eng.prefill([], [(z[:0], z[:0], z[:0], None, None)])[0] == []


def test_binding_refuses():
    D = _D()
    x = R.inputs("gdn", [20, 12], 2, 64, 64)
    c = P.Call("gdn", x, backward=True)
    c.build()
    with pytest.raises(ValueError):
        D.dl_prefill(c.desc, c.S_in, c.S_out, c.tok, c.o.bfloat16(), c.tables, c.ws)
    with pytest.raises(ValueError):
        D.dl_prefill(c.desc, c.S_in[:1], c.S_out, c.tok, c.o, c.tables, c.ws)
    with pytest.raises(ValueError):
        D.dl_prefill(c.desc, c.S_in, c.S_out, c.tok, c.o, D.ChunkTables(2, 31), c.ws)
    with pytest.raises(ValueError):
        D.dl_prefill(c.desc, c.S_in, c.S_out, c.tok, c.o, c.tables, None)
    with pytest.raises(D.DeltaLogError):
        D.dl_prefill(c.desc, c.S_in, c.S_out, c.tok, c.o, c.tables, c.ws[:256])
    with pytest.raises(ValueError):
        D.dl_chunk_tables(c.lens.long(), c.tables)
    with pytest.raises(ValueError):
        D.Grads(c.desc, c.tok, c.S_in[:, :1])


# ------------------------------------------------------------------ training
@pytest.mark.parametrize("op", R.OPS)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_autograd(op, dtype):
    from paper_2608_15533_amd.sequence import delta_scan
    lens = [33, 0, 12]
    x = R.inputs(op, lens, 2, 64, 64, dtype, seed=11)
    x["slots"] = [0, 1, 2]
    want = R.expected(op, x, grads=True)
    y = {n: x[n].cuda().requires_grad_() for n in R.GRADS if x[n] is not None}
    o, S = delta_scan(op, y["q"], y["k"], y["v"], y.get("lam"), y.get("beta"), y.get("u"), y["S"],
                      torch.tensor(lens, dtype=torch.int32, device="cuda"))
    loss = (o * x["do"].cuda()).sum() + (S * x["dS"].cuda()).sum()
    got = torch.autograd.grad(loss, list(y.values()))
    assert R.rel(o, want["o"]) <= R.tol(dtype)
    for (name, leaf), g in zip(y.items(), got):
        assert g.dtype == leaf.dtype
        assert R.rel(g, want["grads"][R.GRADS[name]]) <= R.tol(g.dtype), name


def test_autograd_of_parts():
    """Only the outputs used, or only the states; no initial state; expanded gradients."""
    from paper_2608_15533_amd.sequence import delta_scan
    x = R.inputs("kda", [40], 2, 64, 64, seed=12)
    leaf = {n: x[n].cuda().requires_grad_() for n in ("q", "k", "v", "lam", "beta")}
    o, S = delta_scan("kda", **leaf)
    (go,) = torch.autograd.grad(o.sum(), leaf["v"], retain_graph=True)
    (gs,) = torch.autograd.grad(S.sum(), leaf["v"])
    x["S"], x["do"], x["dS"] = torch.zeros(1, 2, 64, 64), torch.ones_like(x["v"]), torch.zeros(1, 2, 64, 64)
    assert R.rel(go, R.expected("kda", x, grads=True)["grads"]["dv"]) <= R.TOL_F32
    x["do"], x["dS"] = torch.zeros_like(x["v"]), torch.ones(1, 2, 64, 64)
    assert R.rel(gs, R.expected("kda", x, grads=True)["grads"]["dv"]) <= R.TOL_F32


@pytest.mark.parametrize("op", ["gdn", "kda", "rwkv6"])
def test_gradients_against_differences(op):
    """The kernels' forward pass differenced along the gradient's own direction: with step h
    relative to the input, o and S in fp32 carry TOL_F32 / h of noise at the very most and the
    second difference h^2; h = 1e-2 and a bar of 2e-2 hold both."""
    x = R.inputs(op, [45], 2, 64, 64, seed=13)
    c = P.Call(op, x, backward=True)
    c.build()
    c.forward()
    c.backward()
    names = [n for n in R.GRADS if c.x[n] is not None]
    grads = {n: getattr(c.grads, R.GRADS[n]).clone() for n in names}

    def loss():
        c.forward()
        return ((c.o.double() * c.x["do"].double()).sum()
                + (c.S_out.double() * c.x["dS"].double()).sum()).item()

    for n in names:
        g, keep = grads[n], c.x[n].clone()
        h = 1e-2 * keep.norm() / g.norm()
        c.x[n].copy_(keep + h * g)
        up = loss()
        c.x[n].copy_(keep - h * g)
        down = loss()
        c.x[n].copy_(keep)
        want = (g.double() ** 2).sum().item()
        assert abs((up - down) / (2 * h.item()) - want) <= 2e-2 * want, n


# ------------------------------------------------------------------ ways of calling
def test_in_place_and_repeated_calls_agree():
    x = R.inputs("kda", [70, 1, 33], 3, 128, 128, BF16, seed=14)
    c = P.Call("kda", x, backward=True)
    c.build()
    c.forward()
    c.backward()
    first = [t.clone() for t in (c.o, c.S_out, c.grads.dq, c.grads.dk, c.grads.dlam, c.grads.dS)]
    c.ws.fill_(0xff)
    c.forward()
    c.backward()
    for a, b in zip(first, (c.o, c.S_out, c.grads.dq, c.grads.dk, c.grads.dlam, c.grads.dS)):
        assert torch.equal(a, b)
    S = c.x["S"].clone()
    c.D.dl_prefill(c.desc, S, S, c.tok, c.o, c.tables, c.ws)
    assert torch.equal(S, c.S_out)


def test_gradient_without_states():
    """No initial states and no gradient of them, no gradient of the final states."""
    x = R.inputs("gdn", [50], 2, 64, 64, seed=15)
    want = R.expected("gdn", x, grads=True, zero_start=True, dS=False)
    c = P.Call("gdn", x, backward=True, zero_start=True)
    c.grads = c.D.Grads(c.desc, c.tok)
    c.build()
    c.backward(dS=False)
    want["grads"].pop("dS")
    P.check_grads(c, want)


def test_a_sequence_does_not_depend_on_its_neighbours():
    """The same sequence alone, first, and last in a batch: the same bits in o and S."""
    lens = [50, 3, 90]
    x = R.inputs("gla", lens, 2, 64, 64, seed=16)
    c = P.Call("gla", x)
    c.build()
    c.forward()
    for i, (a, n) in enumerate(zip([0, 50, 53], lens)):
        one = {k: None if x[k] is None or k == "u" else x[k][a:a + n] for k in ("q", "k", "v", "lam", "do")}
        one.update(beta=None, u=None, S=x["S"][x["slots"][i]][None], dS=None, lens=[n], slots=[0])
        d = P.Call("gla", one)
        d.build()
        d.forward()
        assert torch.equal(d.o, c.o[a:a + n])
        assert torch.equal(d.S_out[0], c.S_out[x["slots"][i]])


def test_not_a_number_stays_in_its_sequence_and_head():
    x = R.inputs("gdn", [40, 40, 40], 3, 64, 64, seed=17)
    c = P.Call("gdn", x, backward=True)
    c.build()
    c.forward()
    c.backward()
    clean = [t.clone() for t in (c.o, c.S_out, c.grads.dq, c.grads.dlam, c.grads.dS)]
    c.x["v"][45, 1, 3] = float("nan")
    c.x["k"][77, 1, 0] = float("inf")
    c.forward()
    c.backward()
    mid = c.x["slots"][1]
    for a, b in zip(clean, (c.o, c.S_out, c.grads.dq, c.grads.dlam, c.grads.dS)):
        a, b = a.clone(), b.clone()
        if a.dim() == 4:
            a[mid, 1] = b[mid, 1] = 0
        else:
            a[40:80, 1] = b[40:80, 1] = 0
        assert torch.equal(a, b)


@pytest.mark.parametrize("op", ["gdn", "kda", "gla", "rwkv6"])
def test_gates_of_zero_forget(op):
    """A log-decay of -inf (a document's border inside a sequence) starts again from nothing."""
    x = R.inputs(op, [60], 2, 64, 64, seed=18)
    x["lam"][0] = x["lam"][25] = x["lam"][26] = x["lam"][59] = -float("inf")
    y = dict(x, lam=x["lam"].clamp(min=-800.0))           # e^-800 is 0 in 64 bits too
    want = R.expected(op, y, grads=True)
    c = P.Call(op, x, backward=True)
    c.build()
    c.forward()
    c.backward()
    P.check_forward(c, want)
    P.check_grads(c, want, strong=True)


def test_other_streams_and_two_at_once():
    """Two calls on two streams with workspaces of their own, and one given by handle."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    calls, wants = [], []
    for i, op in enumerate(("gdn", "rwkv6")):
        x = R.inputs(op, [300, 20], 4, 64, 64, seed=30 + i)
        wants.append(R.expected(op, x, grads=True))
        calls.append(P.Call(op, x, backward=True, stream=streams[i] if i else streams[i].cuda_stream))
    torch.cuda.synchronize()
    for c in calls:
        c.build()
    for c in calls:
        c.forward()
    for c in calls:
        c.backward()
    for s in streams:
        s.synchronize()
    for c, want in zip(calls, wants):
        P.check_forward(c, want)
        P.check_grads(c, want)


@pytest.mark.parametrize("op", ["gdn", "rwkv6"])
def test_capture_and_replay(op):
    """Tables, forward and backward in one graph, replayed on other lengths and inputs with the
    same buffers, eager work in between; every replay equals the eager calls bit for bit."""
    x = R.inputs(op, [64, 30, 1], 2, 64, 128, BF16, seed=40)
    c = P.Call(op, x, backward=True)
    N = c.N

    def everything():
        c.build()
        c.forward()
        c.backward()

    everything()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        everything()
    results = lambda: [t for t in (c.o, c.S_out, c.grads.dq, c.grads.dk, c.grads.dv,  # noqa: E731
                                   c.grads.dlam, c.grads.dS, c.grads.du) if t is not None]
    for i, lens in enumerate(([64, 30, 1], [1, 0, 94], [31, 32, 32], [0, 95, 0])):
        assert sum(lens) == N
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.x["v"].copy_(R.inputs(op, [N], 2, 64, 128, BF16, seed=50 + i)["v"])
        everything()
        want = [t.clone() for t in results()]
        for t in results():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, results()):
            assert torch.equal(a, b)


def test_long_offsets():
    """Token rows past 2^31 elements of the packed buffers: the last sequence of a batch whose
    earlier rows nobody reads (empty middle, one long run of rows skipped by a first sequence)."""
    D = _D()
    H, d, n = 64, 128, 270000                            # n H d = 2.2e9 elements of q
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GiB")
    desc = D.make_desc("retnet", 2, H, d, d, 1, "bf16")
    q = torch.zeros((n, H, d), dtype=BF16, device="cuda")
    k, v = torch.zeros_like(q), torch.zeros_like(q)
    o = torch.zeros_like(q)
    lam = torch.full((n, H), -0.01, device="cuda")
    x = R.inputs("retnet", [40], H, d, d, BF16, seed=60)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        t[n - 40:] = x[name].cuda()
    lam[n - 40:] = x["lam"].cuda()
    tables = D.ChunkTables(2, n)
    D.dl_chunk_tables(torch.tensor([n - 40, 40], dtype=torch.int32, device="cuda"), tables)
    S = torch.zeros((2, H, d, d), device="cuda")
    ws = D.prefill_workspace(desc, 2, n)
    D.dl_prefill(desc, None, S, D.Token(desc, n, q, k, v, lam), o, tables, ws)
    x["S"] = torch.zeros(1, H, d, d)
    want = R.expected("retnet", x)
    assert R.rel(o[n - 40:], want["o"]) <= R.TOL_BF16
    assert R.rel(S[1], want["S"][0]) <= R.TOL_F32
    assert torch.all(S[0] == 0)
