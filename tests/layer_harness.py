"""Runs the operators around a recurrence on ``layer_reference`` inputs.  Not collected by pytest."""

import torch

import layer_reference as R

FILL = 7.0                                     # what outputs hold before a call


def device(x):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in x.items()}


def wide(t, left=8, right=16):
    """The same rows as columns of a wider tensor, whose other columns are NaN."""
    out = torch.full((t.shape[0], left + t.shape[1] + right), float("nan"), dtype=t.dtype, device=t.device)
    out[:, left:left + t.shape[1]] = t
    return out[:, left:left + t.shape[1]]


class Packed:
    """A batch of packed sequences through the convolution or the scan: tables, buffers, calls."""

    def __init__(self, op, x, act="silu", zero_start=False, strided=False, stream=None):
        from paper_2608_15533_amd import deltalog as D
        self.D, self.op, self.x = D, op, device(x)
        y = self.x
        B, self.n = y["s"].shape[0], len(y["lens"])
        self.N, ch = y["x"].shape
        inp = "bf16" if y["x"].dtype == torch.bfloat16 else "f32"
        put = wide if strided else lambda t: t
        self.wide = put
        if op == "conv":
            self.desc = D.make_conv_desc(B, ch, y["w"].shape[1], inp, act)
            self.rows = D.ConvRows(self.desc, self.N, put(y["x"]), y["w"], y["bias"])
            self.ws = D.conv_workspace(self.desc, self.n, self.N)
            self.grads = D.ConvGrads(self.desc, self.rows, y["s"])
        else:
            self.desc = D.make_ssm_desc(B, ch, y["A"].shape[1], inp)
            self.rows = D.SsmRows(self.desc, self.N, put(y["x"]), put(y["dt"]), y["A"], put(y["B"]),
                                  put(y["C"]), skip=y["skip"], dt_bias=y["bias"],
                                  z=None if y["z"] is None else put(y["z"]))
            self.ws = D.ssm_workspace(self.desc, self.n, self.N, backward=True)
            self.grads = D.SsmGrads(self.desc, self.rows, y["s"])
        self.ws.fill_(0xff)                    # NaN wherever something unwritten is read
        self.tables = D.ChunkTables(self.n, self.N, num_slots=B)
        self.lens = torch.tensor(y["lens"], dtype=torch.int32, device="cuda")
        self.slots = torch.tensor(y["slots"], dtype=torch.int32, device="cuda")
        self.s_in = None if zero_start else y["s"]
        self.y = torch.full((self.N, ch), FILL, dtype=y["x"].dtype, device="cuda")
        self.s_out = torch.full_like(y["s"], FILL)
        self.stream = stream

    def build(self):
        self.D.dl_chunk_tables(self.lens, self.tables, slots=self.slots, stream=self.stream)

    def forward(self, s_out=None):
        s_out = self.s_out if s_out is None else s_out
        if self.op == "conv":
            self.D.dl_conv_prefill(self.desc, self.s_in, s_out, self.rows, self.y, self.tables,
                                   stream=self.stream)
        else:
            self.D.dl_ssm_prefill(self.desc, self.s_in, s_out, self.rows, self.y, self.tables, self.ws,
                                  stream=self.stream)

    def backward(self, ds=True):
        call = self.D.dl_conv_backward if self.op == "conv" else self.D.dl_ssm_backward
        call(self.desc, self.s_in, self.rows, self.x["dy"], self.x["ds"] if ds else None, self.grads,
             self.tables, self.ws, stream=self.stream)

    def results(self):
        g = self.grads
        names = ("dx", "dw", "dbias", "ds") if self.op == "conv" else (
            "dx", "ddt", "dA", "dB", "dC", "dskip", "dbias", "dz", "ds")
        out = {"y": self.y, "s": self.s_out}
        out.update({k: getattr(g, k) for k in names if getattr(g, k) is not None})
        return out


def run(op, x, act="silu", backward=True, zero_start=False, final_grad=True, strided=False):
    c = Packed(op, x, act, zero_start, strided)
    c.build()
    c.forward()
    if backward:
        c.backward(final_grad)
    return c


def check(c, want):
    """Every output and gradient against 64 bits; what belongs to nobody stays as it was."""
    x, N = c.x, sum(c.x["lens"])
    t = lambda y: R.tol(c.op, y.dtype)  # noqa: E731
    used = x["slots"]
    rest = [s for s in range(x["s"].shape[0]) if s not in used]
    y, s = want["out"]
    assert R.rel(c.y[:N], y) <= t(c.y), f"y {R.rel(c.y[:N], y):.2e}"
    assert torch.all(c.y[N:] == FILL), "rows behind the last sequence were written"
    assert R.rel(c.s_out[used], s[used]) <= t(c.s_out), f"s {R.rel(c.s_out[used], s[used]):.2e}"
    assert torch.all(c.s_out[rest] == FILL), "a slot without a sequence was written"
    for k, ref in want["grads"].items():
        got = getattr(c.grads, "d" + k)
        if k == "s":
            assert torch.all(got[rest] == 0), "gradient of a slot without a sequence"
            got, ref = got[used], ref[used]
        elif got.shape[0] == c.N and k not in ("w", "bias", "A", "skip"):
            assert torch.all(got[N:] == 0), f"d{k}: rows behind the last sequence"
            got = got[:N]
        assert R.rel(got, ref) <= t(got), f"d{k} {R.rel(got, ref):.2e}"
