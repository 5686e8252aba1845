"""The operators around a recurrence as they are used: layers trained through autograd, prompts followed
by single tokens, capture and replay, several streams."""

import pytest
import torch

import layer_harness as L
import layer_reference as R
import sequence_reference as Q

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def leaves(tree):
    return {k: v.detach().cuda().requires_grad_(v.is_floating_point()) if torch.is_tensor(v) else v
            for k, v in tree.items()}


# ------------------------------------------------------------------ a delta-rule layer
# conv (q, k, v side by side) -> norm and rotation of q, k, shared by two value heads each -> recurrence
H, REP, DK, ROT = 2, 2, 64, 32
QK, V = H * DK, H * REP * DK


def gdn_inputs(lens, seed, dtype=F32):
    z, N = R._normal(seed), sum(lens)
    return {"x": z(N, 2 * QK + V).to(dtype), "w": (0.5 * z(2 * QK + V, 4)).to(F32),
            "lam": -0.1 * z(N, H * REP).abs().to(F32), "beta": torch.sigmoid(z(N, H * REP)).to(F32),
            "wq": (1 + 0.2 * z(DK)).to(F32), "wk": (1 + 0.2 * z(DK)).to(F32),
            "pos": torch.cat([torch.arange(n) for n in lens]).to(torch.int32),
            "freq": (100.0 ** (-torch.arange(ROT // 2) / (ROT / 2))).to(F32),
            "do": z(N, H * REP, DK).to(dtype)}


def gdn_reference(x, lens):
    v = {k: t.double().requires_grad_(t.is_floating_point()) if torch.is_tensor(t) else t for k, t in x.items()}
    n = len(lens)
    zero = torch.zeros(n, 3, 2 * QK + V, dtype=torch.float64)
    y, s = R.conv({"x": v["x"], "w": v["w"], "bias": None, "s": zero}, lens, range(n), "silu")
    q, k = R.qk({"q": y[:, :QK].unflatten(1, (H, DK)), "k": y[:, QK:2 * QK].unflatten(1, (H, DK)),
                 "wq": v["wq"], "wk": v["wk"], "pos": x["pos"], "freq": x["freq"]}, "rms", "halves", ROT, REP,
                DK ** -0.5)
    S0 = torch.zeros(n, H * REP, DK, DK, dtype=torch.float64)
    # keys of unit length keep the recurrence from growing
    o, S = Q.scan("gdn", lens, range(n), q, k / DK ** 0.5, y[:, 2 * QK:].unflatten(1, (H * REP, DK)),
                  v["lam"], v["beta"], None, S0)
    grads = torch.autograd.grad((o * x["do"].double()).sum(), [v[k] for k in ("x", "w", "lam", "beta", "wq", "wk")])
    return o.detach(), S.detach(), s.detach(), dict(zip(("x", "w", "lam", "beta", "wq", "wk"), grads))


@pytest.mark.parametrize("dtype,bar", [(F32, 2 * Q.TOL_F32), (BF16, 6 * Q.TOL_BF16)], ids=["f32", "bf16"])
def test_a_delta_rule_layer_trains(dtype, bar):
    """fp32: the recurrence's own tolerance twice, for errors that it receives and passes on.  bf16: the
    roundings of the convolution, the norm, keys' scale, the output and their gradients on the way back,
    2^-8 each, six on the longest path."""
    from paper_2608_15533_amd import deltalog as D
    from paper_2608_15533_amd import sequence as M
    lens = [70, 0, 33]
    x = gdn_inputs(lens, 1, dtype)
    want_o, want_S, want_s, want = gdn_reference(x, lens)
    t = leaves(x)
    tables = D.ChunkTables(3, sum(lens))
    D.dl_chunk_tables(i32(lens), tables)
    qk, s1 = M.short_conv(t["x"][:, :2 * QK], t["w"][:2 * QK], lens=tables)
    v, s2 = M.short_conv(t["x"][:, 2 * QK:], t["w"][2 * QK:], lens=tables)
    q, k = M.qk_norm(qk[:, :QK].unflatten(1, (H, DK)), qk[:, QK:].unflatten(1, (H, DK)), t["pos"], t["freq"],
                     t["wq"], t["wk"], norm="rms", turn="halves", rep=REP, q_scale=DK ** -0.5, tables=tables)
    o, S = M.delta_scan("gdn", q, k / DK ** 0.5, v.unflatten(1, (H * REP, DK)), t["lam"], t["beta"], lens=i32(lens))
    got = torch.autograd.grad((o * t["do"].detach()).sum(), [t[n] for n in want])
    assert R.rel(o, want_o) <= bar and R.rel(S, want_S) <= bar
    assert torch.equal(torch.cat([s1, s2], 2).double().cpu(), want_s)
    for (name, ref), g in zip(want.items(), got):
        assert g.dtype == t[name].dtype
        assert R.rel(g, ref) <= bar, f"{name} {R.rel(g, ref):.2e}"


def test_a_delta_rule_layer_answers():
    """A prompt, then single tokens, against the layer over the whole sequence: the steps' convolution
    from the prompt's inputs, norms of single rows at their positions, the decode step's log."""
    from paper_2608_15533_amd import deltalog as D
    lens, steps = [37, 50], 7
    x = gdn_inputs(lens, 2)
    o_ref, _, _, _ = gdn_reference(x, lens)
    x = L.device(x)
    prompt = [n - steps for n in lens]
    rows = torch.cat([torch.arange(0, prompt[0]), torch.arange(lens[0], lens[0] + prompt[1])]).cuda()
    conv = D.make_conv_desc(2, 2 * QK + V, 4, "f32")
    norm = D.make_qk_desc(H, DK, "rms", "halves", ROT, REP, "f32", q_scale=DK ** -0.5)
    rec = D.make_desc("gdn", 2, H * REP, DK, DK, 4, "f32")
    s = torch.zeros(2, 3, 2 * QK + V, device="cuda")
    state = D.DeltaLogState(rec)

    def through(idx, convolve):
        n = idx.numel()
        y = torch.empty(n, 2 * QK + V, device="cuda")
        convolve(D.ConvRows(conv, n, x["x"][idx], x["w"]), y)
        q, k = (torch.empty(n, H * REP, DK, device="cuda") for _ in range(2))
        D.dl_qk_norm(norm, D.QkRows(norm, n, y[:, :QK].unflatten(1, (H, DK)),
                                    y[:, QK:2 * QK].unflatten(1, (H, DK)), x["pos"][idx], x["freq"], x["wq"],
                                    x["wk"]), q, k)
        v = y[:, 2 * QK:].unflatten(1, (H * REP, DK)).contiguous()
        return D.Token(rec, n, q, k / DK ** 0.5, v, x["lam"][idx], x["beta"][idx])

    tables = D.ChunkTables(2, sum(prompt))
    D.dl_chunk_tables(i32(prompt), tables)
    tok = through(rows, lambda r, y: D.dl_conv_prefill(conv, None, s, r, y, tables))
    o = torch.empty(sum(prompt), H * REP, DK, device="cuda")
    D.dl_prefill(rec, None, state.S, tok, o, tables, D.prefill_workspace(rec, 2, sum(prompt)))
    assert R.rel(o, o_ref[rows.cpu()]) <= 2 * Q.TOL_F32
    for t in range(steps):
        idx = torch.tensor([prompt[0] + t, lens[0] + prompt[1] + t], device="cuda")
        tok = through(idx, lambda r, y: D.dl_conv_step(conv, s, s, r, y))
        one = torch.empty(2, H * REP, DK, device="cuda")
        D.dl_append_step(rec, state, tok, one)
        assert R.rel(one, o_ref[idx.cpu()]) <= 2 * Q.TOL_F32


# ------------------------------------------------------------------ a selective-scan layer
def mixer_inputs(lens, D, S, seed, dtype=F32):
    """Columns of one projection: x, z, dt, B, C."""
    z, N = R._normal(seed), sum(lens)
    p = z(N, 3 * D + 2 * S)
    p[:, 2 * D:3 * D] -= 2
    return {"p": p.to(dtype), "w": (0.5 * z(D, 4)).to(F32), "bias": (0.2 * z(D)).to(F32),
            "A": -(torch.arange(1, S + 1) * torch.exp(0.2 * z(D, S))).to(F32), "skip": (1 + 0.2 * z(D)).to(F32),
            "dt_bias": (0.2 * z(D)).to(F32), "dy": z(N, D).to(dtype)}


MIXER = ("p", "w", "bias", "A", "skip", "dt_bias")


def mixer_reference(x, lens, D, S):
    v = {k: x[k].double().requires_grad_() for k in MIXER}
    n = len(lens)
    y, s = R.conv({"x": v["p"][:, :D], "w": v["w"], "bias": v["bias"],
                   "s": torch.zeros(n, 3, D, dtype=torch.float64)}, lens, range(n), "silu")
    cut = v["p"][:, 2 * D:].split([D, S, S], 1)
    y, h = R.ssm({"x": y, "dt": cut[0], "A": v["A"], "B": cut[1], "C": cut[2], "skip": v["skip"],
                  "bias": v["dt_bias"], "z": v["p"][:, D:2 * D],
                  "s": torch.zeros(n, D, S, dtype=torch.float64)}, lens, range(n))
    grads = torch.autograd.grad((y * x["dy"].double()).sum(), [v[k] for k in MIXER])
    return y.detach(), h.detach(), s.detach(), dict(zip(MIXER, grads))


@pytest.mark.parametrize("dtype,bar", [(F32, 2 * R.TOL["ssm"]), (BF16, 2 * R.TOL["ssm"] + 4 * 2.0 ** -8)],
                         ids=["f32", "bf16"])
@pytest.mark.parametrize("S", [16, 32, 64])
def test_a_selective_scan_layer_trains(dtype, bar, S):
    """bf16: the convolution's output and its gradient, the scan's output and an input's gradient are
    rounded on the longest path, 2^-8 each."""
    from paper_2608_15533_amd import sequence as M
    lens, D = [90, 0, 1, 40], 72
    x = mixer_inputs(lens, D, S, 3, dtype)
    want_y, want_h, want_s, want = mixer_reference(x, lens, D, S)
    t = leaves(x)
    y, s = M.short_conv(t["p"][:, :D], t["w"], t["bias"], lens=i32(lens))
    dt, B, C = t["p"][:, 2 * D:].split([D, S, S], 1)
    y, h = M.selective_scan(y, dt, t["A"], B, C, t["skip"], t["dt_bias"], t["p"][:, D:2 * D], lens=i32(lens))
    got = torch.autograd.grad((y * t["dy"].detach()).sum(), [t[k] for k in MIXER])
    assert R.rel(y, want_y) <= bar and R.rel(h, want_h) <= bar
    assert torch.equal(s.double().cpu(), want_s)
    for (name, ref), g in zip(want.items(), got):
        assert R.rel(g, ref) <= bar, f"{name} {R.rel(g, ref):.2e}"


def test_a_selective_scan_layer_answers():
    """A prompt in two parts, then single tokens, against the layer over the whole sequence."""
    from paper_2608_15533_amd import deltalog as D
    lens, ch, S, steps = [60, 45], 72, 16, 6
    x = mixer_inputs(lens, ch, S, 4)
    y_ref, h_ref, s_ref, _ = mixer_reference(x, lens, ch, S)
    x = L.device(x)
    conv, scan = D.make_conv_desc(2, ch, 4, "f32"), D.make_ssm_desc(2, ch, S, "f32")
    s, h = torch.zeros(2, 3, ch, device="cuda"), torch.zeros(2, ch, S, device="cuda")

    def through(idx, tables=None):
        n, p = idx.numel(), x["p"][idx]
        u, y = (torch.empty(n, ch, device="cuda") for _ in range(2))
        c = D.ConvRows(conv, n, p[:, :ch], x["w"], x["bias"])
        dt, B, C = p[:, 2 * ch:].split([ch, S, S], 1)
        if tables is None:
            D.dl_conv_step(conv, s, s, c, u)
        else:
            D.dl_conv_prefill(conv, s, s, c, u, tables)
        r = D.SsmRows(scan, n, u, dt, x["A"], B, C, x["skip"], x["dt_bias"], p[:, ch:2 * ch])
        if tables is None:
            D.dl_ssm_step(scan, h, h, r, y)
        else:
            D.dl_ssm_prefill(scan, h, h, r, y, tables, D.ssm_workspace(scan, 2, n))
        assert R.rel(y, y_ref[idx.cpu()]) <= 2 * R.TOL["ssm"]

    at = [0, lens[0]]
    for part in ([20, 39], [lens[0] - 20 - steps, lens[1] - 39 - steps]):
        idx = torch.cat([torch.arange(a, a + n) for a, n in zip(at, part)]).cuda()
        tables = D.ChunkTables(2, sum(part))
        D.dl_chunk_tables(i32(part), tables)
        through(idx, tables)
        at = [a + n for a, n in zip(at, part)]
    for t in range(steps):
        through(torch.tensor([at[0] + t, at[1] + t], device="cuda"))
    assert R.rel(h, h_ref) <= 2 * R.TOL["ssm"] and torch.equal(s.double().cpu(), s_ref)


# ------------------------------------------------------------------ autograd
def test_autograd_of_parts():
    """Only the outputs used, or only the states; no states given; expanded gradients."""
    from paper_2608_15533_amd import sequence as M
    x = R.ssm_inputs([50], 64, 16, seed=5)
    t = leaves({k: x[k] for k in ("x", "dt", "A", "B", "C", "z", "skip", "bias", "s")})
    y, h = M.selective_scan(t["x"], t["dt"], t["A"], t["B"], t["C"], t["skip"], t["bias"], t["z"], t["s"])
    (gy,) = torch.autograd.grad(y.sum(), t["B"], retain_graph=True)
    (gh,) = torch.autograd.grad(h.sum(), t["B"])
    one = dict(x, dy=torch.ones_like(x["x"]), ds=torch.zeros_like(x["s"]))
    assert R.rel(gy, R.ssm_expected(one)["grads"]["B"]) <= R.TOL["ssm"]
    one = dict(x, dy=torch.zeros_like(x["x"]), ds=torch.ones_like(x["s"]))
    assert R.rel(gh, R.ssm_expected(one)["grads"]["B"]) <= R.TOL["ssm"]
    c = R.conv_inputs([50], 64, 3, seed=6)
    t = leaves({k: c[k] for k in ("x", "w")})
    y, s = M.short_conv(t["x"], t["w"])
    (gs,) = torch.autograd.grad(s.sum(), t["x"], retain_graph=True)
    assert torch.equal(gs.cpu(), torch.cat([torch.zeros(48, 64), torch.ones(2, 64)]))
    (gy,) = torch.autograd.grad(y.sum(), t["w"])
    one = dict(c, bias=None, dy=torch.ones_like(c["x"]))
    assert R.rel(gy, R.conv_expected(one, zero_start=True, final_grad=False)["grads"]["w"]) <= R.TOL["conv"]


@pytest.mark.parametrize("op", ["conv", "ssm"])
def test_gradients_against_differences(op):
    """The kernels' forward pass differenced along the gradient's own direction, as for the recurrence:
    step 1e-2 of the input, noise TOL / 1e-2 and the second difference 1e-4 at most; bar 2e-2.  No entry of
    A moves by more than 0.1: decays are exponentials of A, and with the norm's step one of -1 would move by
    1.06 and the state grow (in 64 bits the difference is then 10 times the gradient, with 0.1 0.5% off)."""
    make = R.conv_inputs if op == "conv" else R.ssm_inputs
    names = ("x", "w", "bias", "s") if op == "conv" else ("x", "dt", "A", "B", "C", "skip", "bias", "z", "s")
    x = make([45, 20], 64, 4 if op == "conv" else 16, seed=7)
    c = L.run(op, x)
    grads = {n: getattr(c.grads, "d" + n).clone() for n in names}

    def loss():
        c.forward()
        return ((c.y.double() * c.x["dy"].double()).sum() + (c.s_out.double() * c.x["ds"].double()).sum()).item()

    for n in names:
        g, keep = grads[n], c.x[n].clone()
        h = 1e-2 * keep.norm() / g.norm()
        if n == "A":
            h = torch.minimum(h, 0.1 / g.abs().max())
        c.x[n].copy_(keep + h * g)
        up = loss()
        c.x[n].copy_(keep - h * g)
        down = loss()
        c.x[n].copy_(keep)
        want = (g.double() ** 2).sum().item()
        assert abs((up - down) / (2 * h.item()) - want) <= 2e-2 * want, n


@pytest.mark.parametrize("tokens", [0, 1, 10, 32, 33])
def test_short_batches_through_autograd(tokens):
    """Few tokens need no workspace; without any, states pass through and parameters get nothing."""
    from paper_2608_15533_amd import sequence as M
    lens = [tokens, 0]
    x = R.ssm_inputs(lens, 72, 16, seed=11)
    x["slots"] = [0, 1]
    want = R.ssm_expected(x)
    t = leaves({k: x[k] for k in ("x", "dt", "A", "B", "C", "skip", "bias", "z", "s")})
    y, h = M.selective_scan(t["x"], t["dt"], t["A"], t["B"], t["C"], t["skip"], t["bias"], t["z"], t["s"], i32(lens))
    got = torch.autograd.grad([y, h], list(t.values()), [x["dy"].cuda(), x["ds"].cuda()])
    assert R.rel(y, want["out"][0]) <= R.TOL["ssm"] and R.rel(h, want["out"][1]) <= R.TOL["ssm"]
    for k, g in zip(t, got):
        assert R.rel(g, want["grads"][k]) <= R.TOL["ssm"], k
    c = R.conv_inputs(lens, 72, 4, seed=12)
    c["slots"] = [0, 1]
    want = R.conv_expected(c)
    t = leaves({k: c[k] for k in ("x", "w", "bias", "s")})
    y, s = M.short_conv(t["x"], t["w"], t["bias"], t["s"], i32(lens))
    got = torch.autograd.grad([y, s], list(t.values()), [c["dy"].cuda(), c["ds"].cuda()])
    assert R.rel(y, want["out"][0]) <= R.TOL["conv"] and torch.equal(s.double().cpu(), want["out"][1])
    for k, g in zip(t, got):
        assert R.rel(g, want["grads"][k]) <= R.TOL["conv"], k


# ------------------------------------------------------------------ ways of calling
@pytest.mark.parametrize("op", ["conv", "ssm"])
def test_capture_and_replay(op):
    """Tables, forward and backward in one graph, replayed on other lengths and inputs with the same
    buffers, eager work in between; every replay equals the eager calls bit for bit."""
    make = R.conv_inputs if op == "conv" else R.ssm_inputs
    width = 4 if op == "conv" else 16
    x = make([200, 30, 1], 136, width, BF16, seed=8)
    c = L.Packed(op, x)

    def everything():
        c.build()
        c.forward()
        c.backward()

    everything()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        everything()
    for i, lens in enumerate(([200, 30, 1], [1, 0, 230], [31, 100, 100], [0, 231, 0])):
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.x["x"].copy_(make([231], 136, width, BF16, seed=9 + i)["x"])
        everything()
        want = {k: v.clone() for k, v in c.results().items()}
        for v in c.results().values():
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        for k, v in c.results().items():
            assert torch.equal(v, want[k]), k


def test_norm_in_a_graph():
    from test_gpu_qk_norm import Call
    c = Call(R.qk_inputs(40, 3, 64, 64, 2, BF16, seed=10), "rms", "halves", 64, 2)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward()
        c.backward()
    for i in range(3):
        c.x["q"].copy_(R.qk_inputs(40, 3, 64, 64, 2, BF16, seed=20 + i)["q"])
        c.forward()
        c.backward()
        want = {k: v.clone() for k, v in c.results().items()}
        for v in c.results().values():
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, want[k]) for k, v in c.results().items())


@pytest.mark.parametrize("op", ["conv", "ssm", "qk"])
def test_a_training_step_in_a_graph(op):
    """Forward and backward through autograd captured together, leaves that no eager graph holds; every
    replay equals the eager step bit for bit, with eager work of other leaves in between."""
    from paper_2608_15533_amd import sequence as M
    lens = [70, 0, 1, 40]
    make = {"conv": lambda s: R.conv_inputs(lens, 136, 4, BF16, seed=s),
            "ssm": lambda s: R.ssm_inputs(lens, 136, 16, BF16, seed=s),
            "qk": lambda s: R.qk_inputs(sum(lens), 2, 64, 64, 2, BF16, seed=s)}[op]
    names = {"conv": ("x", "w", "bias"), "ssm": ("x", "dt", "A", "B", "C", "skip", "bias", "z"),
             "qk": ("q", "k", "wq", "wk")}[op]

    def step(t, n):
        if op == "conv":
            out = (M.short_conv(t["x"], t["w"], t["bias"], lens=n)[0],)
        elif op == "ssm":
            out = (M.selective_scan(t["x"], t["dt"], t["A"], t["B"], t["C"], t["skip"],
                                    t["bias"], t["z"], lens=n)[0],)
        else:
            out = M.qk_norm(t["q"], t["k"], t["pos"], t["freq"], t["wq"], t["wk"], "rms", "halves",
                            rep=2)
        ones = [torch.full_like(o, 0.5) for o in out]
        return [o.detach() for o in out] + list(torch.autograd.grad(out, [t[k] for k in names], ones))

    n = i32(lens)
    step(leaves(make(0)), n)
    held = leaves(make(1))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(held, n)
    for seed in (1, 2, 3):
        x = make(seed)
        want = step(leaves(x), n)
        with torch.no_grad():
            for k in names:
                held[k].copy_(x[k])
            if op == "qk":
                held["pos"].copy_(x["pos"])
        for o in got:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        for o, w in zip(got, want):
            assert torch.equal(o, w)


def test_other_streams_and_two_at_once():
    """Calls on two streams with workspaces of their own, one given by handle."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    calls, wants = [], []
    for i, op in enumerate(("conv", "ssm")):
        x = (R.conv_inputs([300, 20], 136, 4, seed=30) if op == "conv" else
             R.ssm_inputs([300, 20], 136, 16, seed=31))
        wants.append(R.conv_expected(x) if op == "conv" else R.ssm_expected(x))
        calls.append(L.Packed(op, x, stream=streams[i] if i else streams[i].cuda_stream))
    torch.cuda.synchronize()
    for step in ("build", "forward", "backward"):
        for c in calls:
            getattr(c, step)()
    for s in streams:
        s.synchronize()
    for c, want in zip(calls, wants):
        L.check(c, want)


def test_long_offsets():
    """Rows past 2^31 elements: the last sequence of a batch whose first is left out (its slot does not
    exist), so that nothing else is read."""
    from paper_2608_15533_amd import deltalog as D
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GiB")
    ch, n = 8192, 270000                                 # 2.2e9 elements
    x = R.conv_inputs([40], ch, 4, BF16, seed=40)
    big = torch.empty((n, ch), dtype=BF16, device="cuda")
    big[n - 40:] = x["x"].cuda()
    y = torch.empty_like(big)
    desc = D.make_conv_desc(2, ch, 4)
    tables = D.ChunkTables(2, n)
    D.dl_chunk_tables(i32([n - 40, 40]), tables, slots=i32([5, 1]))
    s = torch.zeros((2, 3, ch), dtype=BF16, device="cuda")
    rows = D.ConvRows(desc, n, big, x["w"].cuda(), x["bias"].cuda())
    D.dl_conv_prefill(desc, None, s, rows, y, tables)
    want = R.conv_expected(x, zero_start=True, grads=False)
    assert R.rel(y[n - 40:], want["out"][0]) <= R.tol("conv", BF16)
    assert torch.equal(s[1].double().cpu(), want["out"][1][0])
    dx = D.ConvGrads(desc, rows)
    dy = torch.empty_like(big)
    dy[n - 40:] = x["dy"].cuda()
    D.dl_conv_backward(desc, None, rows, dy, None, dx, tables, D.conv_workspace(desc, 2, n))
    want = R.conv_expected(x, zero_start=True, final_grad=False)["grads"]
    assert R.rel(dx.dx[n - 40:], want["x"]) <= R.tol("conv", BF16)
    assert R.rel(dx.dw, want["w"]) <= R.TOL["conv"]
