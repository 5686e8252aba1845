"""Runs dl_chunk_tables, dl_prefill and dl_prefill_backward on ``sequence_reference.inputs``.
Not collected by pytest."""

import torch

import sequence_reference as R


def device(x):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in x.items()}


class Call:
    """One batch on the device: tables, buffers, the calls."""

    def __init__(self, op, x, state="f32", backward=False, zero_start=False, stream=None):
        from paper_2608_15533_amd import deltalog as D
        self.D, self.op, self.x = D, op, device(x)
        y = self.x
        self.N, self.n = y["q"].shape[0], len(y["lens"])
        H, dk, dv = y["q"].shape[1], y["q"].shape[2], y["v"].shape[2]
        inp = "bf16" if y["q"].dtype == torch.bfloat16 else "f32"
        self.desc = D.make_desc(op, y["S"].shape[0], H, dk, dv, 4, inp, state)
        self.tables = D.ChunkTables(self.n, self.N, num_slots=y["S"].shape[0])
        self.lens = torch.tensor(y["lens"], dtype=torch.int32, device="cuda")
        self.slots = torch.tensor(y["slots"], dtype=torch.int32, device="cuda")
        self.tok = D.Token(self.desc, self.N, y["q"], y["k"], y["v"], y["lam"], y["beta"], y["u"])
        self.S_in = None if zero_start else y["S"]
        self.o = torch.full_like(y["v"], 7.0)
        self.S_out = torch.full_like(y["S"], 7.0)
        self.ws = D.prefill_workspace(self.desc, self.n, self.N, backward)
        self.ws.fill_(0xff)                              # NaN wherever something unwritten is read
        self.grads = D.Grads(self.desc, self.tok, y["S"]) if backward else None
        self.stream = stream

    def build(self):
        self.D.dl_chunk_tables(self.lens, self.tables, slots=self.slots, stream=self.stream)

    def forward(self):
        self.D.dl_prefill(self.desc, self.S_in, self.S_out, self.tok, self.o, self.tables,
                          self.ws, stream=self.stream)

    def backward(self, dS=True):
        self.D.dl_prefill_backward(self.desc, self.S_in, self.tok, self.x["do"],
                                   self.x["dS"] if dS else None, self.grads, self.tables,
                                   self.ws, stream=self.stream)


def check_forward(call, want):
    N, x = sum(call.x["lens"]), call.x
    e = R.rel(call.o[:N], want["o"])
    assert e <= R.tol(call.o.dtype), f"o {e:.2e}"
    assert torch.all(call.o[N:] == 7.0), "rows behind the last sequence were written"
    used = x["slots"]
    if used:
        e = R.rel(call.S_out[used], want["S"][used])
        assert e <= R.tol(call.S_out.dtype), f"S {e:.2e}"
    rest = [s for s in range(x["S"].shape[0]) if s not in used]
    assert torch.all(call.S_out[rest] == 7.0), "a slot without a sequence was written"


def check_grads(call, want, strong=False):
    """``strong``: decays that forget within a few tokens.  dlam_t is a sum over the chunk's
    tokens from t on of q dq + k dk' - k dk'', of which then only what crosses t is left: its
    error is measured against those terms, as that of any sum that cancels."""
    N, g = sum(call.x["lens"]), call.grads
    for name, ref in want["grads"].items():
        got = getattr(g, name)
        if name == "dS":
            got, ref = got[call.x["slots"]], ref[call.x["slots"]]
        elif name != "du":
            assert torch.all(got[N:] == 0), f"{name}: rows behind the last sequence"
            got = got[:N]
        e = R.rel(got, ref)
        if name == "dlam" and strong:
            terms = [call.x[a][:N].double().cpu() * want["grads"]["d" + a] for a in ("q", "k")]
            if ref.dim() == 2:
                terms = [t.sum(-1) for t in terms]
            e *= ref.norm().item() / max(t.norm().item() for t in terms + [ref])
        assert e <= R.tol(got.dtype), f"{name} {e:.2e}"
