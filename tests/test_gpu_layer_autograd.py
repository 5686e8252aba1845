"""The torch functions of the operators around a recurrence in a training program: tables filled again while
earlier calls wait for their gradients, other default dtypes."""

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
