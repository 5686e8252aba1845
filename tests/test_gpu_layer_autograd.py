"""The torch functions of the operators around a recurrence in a training program: tables filled again while
earlier calls wait for their gradients, other default dtypes, slots without a sequence, frequencies."""

import pytest
import torch

import layer_harness as L
import layer_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
LEAVES = {"conv": ("x", "w", "bias", "s"), "ssm": ("x", "dt", "A", "B", "C", "skip", "bias", "z", "s"),
          "qk": ("q", "k", "wq", "wk")}
FIRST, SECOND = ([70, 3, 0, 40], [2, 0, 3, 1]), ([10, 50, 23, 5], [0, 3, 1, 2])


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def leaves(x, names):
    return {k: x[k].cuda().requires_grad_() for k in names}


def fill(tables, batch):
    from paper_2608_15533_amd import deltalog as D
    D.dl_chunk_tables(i32(batch[0]), tables, slots=i32(batch[1]))


def call(op, t, x, lens):
    from paper_2608_15533_amd import sequence as M
    if op == "conv":
        return M.short_conv(t["x"], t["w"], t["bias"], t["s"], lens)
    if op == "ssm":
        return M.selective_scan(t["x"], t["dt"], t["A"], t["B"], t["C"], t["skip"], t["bias"], t["z"], t["s"], lens)
    return M.qk_norm(t["q"], t["k"], x["pos"].cuda(), x["freq"].cuda(), t["wq"], t["wk"], "rms", "halves", rep=2,
                     q_scale=0.3, tables=lens)


def make(op, seed, dtype=F32, B=4):
    if op == "conv":
        return R.conv_inputs([113], 72, 4, dtype, B=B, seed=seed)
    if op == "ssm":
        return R.ssm_inputs([113], 72, 16, dtype, B=B, seed=seed)
    return R.qk_inputs(113, 2, 64, 64, 2, dtype, seed=seed)


# ------------------------------------------------------------------ tables filled again
@pytest.mark.parametrize("op", ["conv", "ssm", "qk"])
def test_gradients_are_of_the_calls_own_tables(op):
    """Two batches through one ChunkTables, then the gradients of both: each by the lengths and slots of its
    own forward call (the second leaves rows behind its last sequence)."""
    from paper_2608_15533_amd import deltalog as D
    tables = D.ChunkTables(4, 113)
    calls = []
    for seed, (lens, slots) in enumerate((FIRST, SECOND)):
        x = dict(make(op, seed), lens=lens, slots=slots)
        t = leaves(x, LEAVES[op])
        fill(tables, (lens, slots))
        calls.append((x, t, call(op, t, x, tables)))
    for x, t, out in calls:
        N = sum(x["lens"])
        if op == "qk":
            used = {k: v[:N] if v.shape[0] == 113 else v for k, v in x.items() if torch.is_tensor(v)}
            want = R.qk_expected(used, "rms", "halves", 64, 2, 0.3)["grads"]
            ends = [x["dqo"].cuda(), x["dko"].cuda()]
        else:
            want = (R.conv_expected if op == "conv" else R.ssm_expected)(x)["grads"]
            ends = [x["dy"].cuda(), x["ds"].cuda()]
        got = torch.autograd.grad(out, list(t.values()), ends)
        for (k, leaf), g in zip(t.items(), got):
            if leaf.shape[0] == 113:
                assert torch.all(g[N:] == 0), f"d{k}: rows behind the last sequence"
                g = g[:N]
            assert R.rel(g, want[k]) <= R.TOL[op], f"d{k} {R.rel(g, want[k]):.2e}"


@pytest.mark.parametrize("op", ["conv", "ssm", "qk"])
def test_tables_filled_in_a_graph(op):
    """Two fillings, two forward calls and the first one's gradients captured together: every replay equals
    the eager calls bit for bit, with eager work in between."""
    from paper_2608_15533_amd import deltalog as D
    tables = D.ChunkTables(4, 113)
    lens, slots = [i32(b[0]) for b in (FIRST, SECOND)], [i32(b[1]) for b in (FIRST, SECOND)]

    def step(x, t):
        D.dl_chunk_tables(lens[0], tables, slots=slots[0])
        out = call(op, t, x, tables)
        D.dl_chunk_tables(lens[1], tables, slots=slots[1])
        call(op, t, x, tables)
        return torch.autograd.grad(out, list(t.values()), [torch.full_like(o, 0.5) for o in out])

    def ready(seed):
        x = {k: v.cuda() if torch.is_tensor(v) else v for k, v in make(op, seed, BF16).items()}
        return x, leaves(x, LEAVES[op])

    step(*ready(0))
    x, held = ready(1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(x, held)
    for seed, batch in enumerate((FIRST, ([0, 0, 113, 0], [1, 0, 3, 2]), ([1, 111, 0, 1], [3, 2, 1, 0]))):
        lens[0].copy_(torch.tensor(batch[0]))
        slots[0].copy_(torch.tensor(batch[1]))
        y, t = ready(seed)
        want = step(y, t)
        with torch.no_grad():
            for k in held:
                held[k].copy_(t[k])
            if op == "qk":
                x["pos"].copy_(y["pos"])
        for o in got:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        for k, o, w in zip(held, got, want):
            assert torch.equal(o, w), k


# ------------------------------------------------------------------ default dtypes
@pytest.mark.parametrize("default", [BF16, torch.float64], ids=["bf16", "f64"])
@pytest.mark.parametrize("op", ["conv", "ssm", "qk"])
def test_another_default_dtype(op, default):
    """torch's default dtype is no input: outputs and gradients are bit for bit those under fp32."""
    x = make(op, 1)
    x["lens"] = i32([60, 0, 53, 0])

    def step():
        t = leaves(x, LEAVES[op])
        out = call(op, t, x, None if op == "qk" else x["lens"])
        return out + torch.autograd.grad(out, list(t.values()), [torch.ones_like(o) for o in out])

    want = step()
    torch.set_default_dtype(default)
    try:
        got = step()
    finally:
        torch.set_default_dtype(F32)
    for g, w in zip(got, want):
        assert g.dtype == w.dtype and torch.equal(g, w)


# ------------------------------------------------------------------ slots without a sequence
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("op", ["conv", "ssm"])
@pytest.mark.parametrize("lens,slots", [([70, 0, 43], [4, 0, 2]), ([113], [1]), ([0], [3]), ([], [])], ids=str)
def test_slots_without_a_sequence_pass_through(op, lens, slots, dtype):
    """Tables of more slots than sequences: the other slots' states come back as they were, and so does their
    gradient; without initial states they are zero."""
    from paper_2608_15533_amd import deltalog as D
    x = dict(make(op, 3, dtype, B=5), lens=lens, slots=slots)
    rest = [s for s in range(5) if s not in slots]
    tables = D.ChunkTables(len(lens), 113, num_slots=5)
    fill(tables, (lens, slots))
    t = leaves(x, LEAVES[op])
    y, s = call(op, t, x, tables)
    got = dict(zip(t, torch.autograd.grad([y, s], list(t.values()), [x["dy"].cuda(), x["ds"].cuda()])))
    assert torch.equal(s[rest].cpu(), x["s"][rest])
    assert torch.equal(got["s"][rest].cpu(), x["ds"][rest])
    if lens:
        want = (R.conv_expected if op == "conv" else R.ssm_expected)(x)
        bar = lambda v: R.tol(op, v.dtype)  # noqa: E731
        N = sum(lens)
        assert R.rel(y[:N], want["out"][0]) <= bar(y) and torch.all(y[N:] == 0)
        assert R.rel(s[slots], want["out"][1][slots]) <= bar(s)
        assert R.rel(got["s"][slots], want["grads"]["s"][slots]) <= bar(s)
        for k in t:
            g = got[k][:N] if got[k].shape[0] == 113 else got[k]
            assert k == "s" or R.rel(g, want["grads"][k]) <= bar(g), k
    else:
        assert torch.all(y == 0) and all(torch.all(g == 0) for k, g in got.items() if k != "s")
    _, s = call(op, dict(t, s=None), x, tables)
    assert torch.all(s[rest] == 0)


@pytest.mark.parametrize("op", ["conv", "ssm"])
def test_a_sequence_that_is_left_out_leaves_its_slot(op):
    """A slot that does not exist: its sequence is skipped, every slot that no sequence has passes through."""
    from paper_2608_15533_amd import deltalog as D
    x = make(op, 4, B=3)
    tables = D.ChunkTables(3, 113)
    fill(tables, ([50, 3, 60], [2, 9, 0]))
    t = leaves(x, LEAVES[op])
    y, s = call(op, t, x, tables)
    (g,) = torch.autograd.grad([y, s], [t["s"]], [x["dy"].cuda(), x["ds"].cuda()])
    assert tables.err.item() == 1 and torch.all(y[50:53] == 0)
    assert torch.equal(s[1].cpu(), x["s"][1]) and torch.equal(g[1].cpu(), x["ds"][1])
    assert not torch.equal(s[0].cpu(), x["s"][0]) and not torch.equal(g[0].cpu(), x["ds"][0])


@pytest.mark.parametrize("op", ["conv", "ssm"])
def test_slots_without_a_sequence_in_a_graph(op):
    """Captured forward and backward: replays on other slots equal the eager step bit for bit."""
    from paper_2608_15533_amd import deltalog as D
    tables, lens, slots = D.ChunkTables(2, 113, num_slots=5), i32([70, 43]), i32([3, 1])

    def step(t):
        D.dl_chunk_tables(lens, tables, slots=slots)
        out = call(op, t, None, tables)
        grads = torch.autograd.grad(out, list(t.values()), [torch.full_like(o, 0.5) for o in out])
        return [o.detach() for o in out] + list(grads)

    step(leaves(make(op, 0, BF16, B=5), LEAVES[op]))
    held = leaves(make(op, 1, BF16, B=5), LEAVES[op])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(held)
    for seed, where in enumerate(([3, 1], [0, 4], [2, 3])):
        slots.copy_(torch.tensor(where))
        t = leaves(make(op, seed, BF16, B=5), LEAVES[op])
        want = step(t)
        with torch.no_grad():
            for k in held:
                held[k].copy_(t[k])
        for o in got:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        for o, w in zip(got, want):
            assert torch.equal(o, w)


# ------------------------------------------------------------------ frequencies
def test_frequencies_are_constants():
    """The rotation's frequencies get no gradient, whatever they require; the others' is the same."""
    x = make("qk", 5)
    t = leaves(x, LEAVES["qk"] + ("freq",))
    plain = leaves(x, LEAVES["qk"])
    from paper_2608_15533_amd import sequence as M
    out = M.qk_norm(t["q"], t["k"], x["pos"].cuda(), t["freq"], t["wq"], t["wk"], "rms", "halves", rep=2, q_scale=0.3)
    got = torch.autograd.grad(out, list(t.values()), [torch.ones_like(o) for o in out], allow_unused=True)
    out = call("qk", plain, x, None)
    want = torch.autograd.grad(out, list(plain.values()), [torch.ones_like(o) for o in out])
    assert got[-1] is None and all(torch.equal(g, w) for g, w in zip(got, want))


def test_gradient_buffers_start_from_states_of_the_call():
    """What slots without a sequence hold has the states' type and shape, or is refused."""
    from paper_2608_15533_amd import deltalog as D
    x = L.device(R.conv_inputs([5], 64, 4, BF16, B=3))
    desc = D.make_conv_desc(3, 64, 4)
    rows = D.ConvRows(desc, 5, x["x"], x["w"], x["bias"])
    g = D.ConvGrads(desc, rows, x["s"], x["ds"])
    assert torch.equal(g.ds, x["ds"]) and g.ds.data_ptr() != x["ds"].data_ptr()
    for bad in (x["ds"].float(), x["ds"][:2], x["ds"].cpu()):
        with pytest.raises(ValueError):
            D.ConvGrads(desc, rows, x["s"], bad)
    x = L.device(R.ssm_inputs([5], 64, 16, BF16, B=3))
    desc = D.make_ssm_desc(3, 64, 16)
    rows = D.SsmRows(desc, 5, x["x"], x["dt"], x["A"], x["B"], x["C"])
    assert torch.equal(D.SsmGrads(desc, rows, x["s"], x["ds"]).ds, x["ds"])
    assert D.SsmGrads(desc, rows, None, x["ds"]).ds is None
    for bad in (x["ds"].to(BF16), x["ds"][:2], x["ds"].cpu()):
        with pytest.raises(ValueError):
            D.SsmGrads(desc, rows, x["s"], bad)
