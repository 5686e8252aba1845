"""Entry points of the operators around a recurrence on a host without a GPU: every refusal comes before
any HIP call (fake device addresses, as in test_abi_cpu.py)."""

import ctypes

import pytest
import torch

from paper_2608_15533_amd import deltalog as D

A = 0x10000000
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: only on a host without a GPU")
N = 100


def ref(x):
    return None if x is None else ctypes.byref(x)


def put(x, /, **kw):
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def tables(**kw):
    return put(D.dl_tables(A, A, A, A, A, A), **kw)


# Every call below is in order but for one thing that is looked at last: an output's alignment.
class Conv:
    @staticmethod
    def desc(**kw):
        return put(D.make_conv_desc(4, 64, 4, "bf16"), **kw)

    @staticmethod
    def rows(**kw):
        return put(D.dl_conv_rows(A, 64, A, A), **kw)

    @staticmethod
    def grads(**kw):
        return put(D.dl_conv_grads(A, A, A, A), **kw)

    @classmethod
    def step(cls, d=None, r=None, s_in=A, s_out=A, y=A + 4, slots=A, n=4):
        return D.lib.dl_conv_step(ref(d or cls.desc()), s_in, s_out, ref(r or cls.rows()), y, slots, n, None)

    @classmethod
    def prefill(cls, d=None, r=None, s_in=A, s_out=A, y=A + 4, tb=None, n=4, tokens=N, ws=A, nbytes=1 << 40):
        return D.lib.dl_conv_prefill(ref(d or cls.desc()), s_in, s_out, ref(r or cls.rows()), y,
                                     ref(tb or tables()), n, tokens, None)

    @classmethod
    def backward(cls, d=None, r=None, s_in=A, dy=A, ds=A, g=None, tb=None, n=4, tokens=N, ws=A + 4,
                 nbytes=1 << 40):
        return D.lib.dl_conv_backward(ref(d or cls.desc()), s_in, ref(r or cls.rows()), dy, ds,
                                      ref(g or cls.grads()), ref(tb or tables()), n, tokens, ws, nbytes, None)

    @classmethod
    def need(cls, d, n=4, tokens=N):
        out = ctypes.c_size_t(0)
        rc = D.lib.dl_conv_workspace_bytes(ref(d), n, tokens, ref(out))
        return rc if rc else out.value


class Ssm:
    @staticmethod
    def desc(**kw):
        return put(D.make_ssm_desc(4, 64, 16, "bf16"), **kw)

    @staticmethod
    def rows(**kw):
        return put(D.dl_ssm_rows(A, A, A, A, A, 64, 64, 64, 16, 16, A, A, A), **kw)

    @staticmethod
    def grads(**kw):
        return put(D.dl_ssm_grads(*[A] * 9), **kw)

    @classmethod
    def step(cls, d=None, r=None, s_in=A, s_out=A, y=A + 4, slots=A, n=4):
        return D.lib.dl_ssm_step(ref(d or cls.desc()), s_in, s_out, ref(r or cls.rows()), y, slots, n, None)

    @classmethod
    def prefill(cls, d=None, r=None, s_in=A, s_out=A, y=A + 4, tb=None, n=4, tokens=N, ws=A, nbytes=1 << 40):
        return D.lib.dl_ssm_prefill(ref(d or cls.desc()), s_in, s_out, ref(r or cls.rows()), y,
                                    ref(tb or tables()), n, tokens, ws, nbytes, None)

    @classmethod
    def backward(cls, d=None, r=None, s_in=A, dy=A, ds=A, g=None, tb=None, n=4, tokens=N, ws=A + 4,
                 nbytes=1 << 40):
        return D.lib.dl_ssm_backward(ref(d or cls.desc()), s_in, ref(r or cls.rows()), dy, ds,
                                     ref(g or cls.grads()), ref(tb or tables()), n, tokens, ws, nbytes, None)

    @classmethod
    def need(cls, d, n=4, tokens=N, backward=1):
        out = ctypes.c_size_t(0)
        rc = D.lib.dl_ssm_workspace_bytes(ref(d), n, tokens, backward, ref(out))
        return rc if rc else out.value


class Qk:
    @staticmethod
    def desc(**kw):
        return put(D.make_qk_desc(4, 64, "rms", "halves", 32, 2, "bf16"), **kw)

    @staticmethod
    def rows(**kw):
        return put(D.dl_qk_rows(A, A, 256, 256, A, A, A, A, A), **kw)

    @staticmethod
    def grads(**kw):
        return put(D.dl_qk_grads(A, A, A, A), **kw)

    @classmethod
    def forward(cls, d=None, r=None, q=A, k=A + 4, n=N):
        return D.lib.dl_qk_norm(ref(d or cls.desc()), ref(r or cls.rows()), q, k, n, None)

    @classmethod
    def backward(cls, d=None, r=None, dq=A, dk=A, g=None, n=N, ws=A + 4, nbytes=1 << 40):
        return D.lib.dl_qk_norm_backward(ref(d or cls.desc()), ref(r or cls.rows()), dq, dk,
                                         ref(g or cls.grads()), n, ws, nbytes, None)


def calls(*ops):
    return [f for op in ops for f in (op.step, op.prefill, op.backward)]


EVERY = calls(Conv, Ssm) + [Qk.forward, Qk.backward]
OWNER = {f.__func__: op for op in (Conv, Ssm, Qk) for f in vars(op).values() if isinstance(f, classmethod)
         for f in [getattr(op, f.__func__.__name__)]}


def owner(call):
    return OWNER[call.__func__]


ids = [f"{owner(f).__name__}-{f.__func__.__name__}" for f in EVERY]
every = pytest.mark.parametrize("call", EVERY, ids=ids)


@every
def test_valid_calls_stop_at_the_planted_alignment(call):
    assert call() == D.DL_E_ALIGN


@every
def test_descriptors(call):
    make = owner(call).desc
    assert call(d=make(abi_version=3)) == D.DL_E_VERSION
    assert call(d=make(in_dtype=2)) == D.DL_E_DTYPE
    bad = {
        Conv: [(dict(channels=60), D.DL_E_SHAPE), (dict(channels=0), D.DL_E_SHAPE), (dict(num_slots=0), D.DL_E_SHAPE),
               (dict(channels=(1 << 24) + 8), D.DL_E_SHAPE), (dict(width=1), D.DL_E_UNSUPPORTED),
               (dict(width=5), D.DL_E_UNSUPPORTED), (dict(activation=2), D.DL_E_UNSUPPORTED),
               (dict(activation=-1), D.DL_E_UNSUPPORTED)],
        Ssm: [(dict(channels=60), D.DL_E_SHAPE), (dict(channels=-8), D.DL_E_SHAPE), (dict(num_slots=0), D.DL_E_SHAPE),
              (dict(channels=(1 << 20) + 8), D.DL_E_SHAPE), (dict(states=8), D.DL_E_UNSUPPORTED),
              (dict(states=48), D.DL_E_UNSUPPORTED), (dict(states=128), D.DL_E_UNSUPPORTED)],
        Qk: [(dict(heads=0), D.DL_E_SHAPE), (dict(rep=0), D.DL_E_SHAPE), (dict(heads=40000), D.DL_E_SHAPE),
             (dict(head_dim=96), D.DL_E_UNSUPPORTED), (dict(norm=3), D.DL_E_UNSUPPORTED),
             (dict(turn=3), D.DL_E_UNSUPPORTED), (dict(rot=0), D.DL_E_SHAPE), (dict(rot=24), D.DL_E_SHAPE),
             (dict(rot=80), D.DL_E_SHAPE), (dict(turn=0), D.DL_E_SHAPE), (dict(eps=0.0), D.DL_E_UNSUPPORTED),
             (dict(eps=float("nan")), D.DL_E_UNSUPPORTED)],
    }[owner(call)]
    for kw, code in bad:
        assert call(d=make(**kw)) == code, kw


def test_no_norm_needs_no_eps():
    assert Qk.forward(d=Qk.desc(norm=0, eps=0.0)) == D.DL_E_ALIGN


@every
def test_counts(call):
    assert call(n=-1) == D.DL_E_SHAPE
    op = owner(call)
    none = {Conv: D.dl_conv_rows, Ssm: D.dl_ssm_rows, Qk: D.dl_qk_rows}[op]()
    assert call(n=0, r=none) == D.DL_OK                       # a no-op
    if op is not Qk:
        assert call(n=5) == D.DL_E_SHAPE                      # more rows or sequences than slots
        huge = op.desc(channels=1 << 20, num_slots=1 << 30)
        if call.__func__.__name__ == "step":
            assert call(d=huge, n=1 << 30) == D.DL_E_SHAPE    # the grid
            assert call(slots=None, n=3) == D.DL_E_SHAPE
        else:
            assert call(tokens=-1) == D.DL_E_SHAPE
            assert call(d=huge, tokens=2 ** 31 - 1) == D.DL_E_SHAPE
    else:
        assert call(n=2 ** 31 - 1) == D.DL_E_SHAPE


def test_grids_of_the_sums_over_channels():
    """Few channels, many tokens: more workgroups for the sums of dB and dC than for the gradients."""
    d, r = Ssm.desc(channels=8, states=64), Ssm.rows(b_stride=64, c_stride=64)
    assert Ssm.backward(d=d, r=r, tokens=30_000_000) == D.DL_E_ALIGN
    assert Ssm.backward(d=d, r=r, tokens=60_000_000) == D.DL_E_SHAPE
    assert Ssm.prefill(d=d, r=r, tokens=60_000_000) == D.DL_E_ALIGN


@every
def test_rows(call):
    op = owner(call)
    needed = {Conv: ("x", "w"), Ssm: ("x", "dt", "B", "C", "A"), Qk: ("q", "k", "pos", "freq")}[op]
    big = {Conv: ("x",), Ssm: ("x", "dt", "z", "B", "C"), Qk: ("q", "k")}[op]
    small = {Conv: ("w", "bias"), Ssm: ("A", "skip", "dt_bias"), Qk: ("pos", "freq", "wq", "wk", "used")}[op]
    strides = {Conv: ("x_stride",), Ssm: ("x_stride", "dt_stride", "z_stride", "b_stride", "c_stride"),
               Qk: ("q_stride", "k_stride")}[op]
    for k in needed:
        assert call(r=op.rows(**{k: None})) == D.DL_E_NULL, k
    for k in big:
        assert call(r=op.rows(**{k: A + 8})) == D.DL_E_ALIGN, k
    for k in small:
        assert call(r=op.rows(**{k: A + 2})) == D.DL_E_ALIGN, k
    for k in strides:
        ok = getattr(op.rows(), k)
        for bad in (ok - 8, ok + 4, 0, -ok, D.DL_MAX_STRIDE + 8):
            assert call(r=op.rows(**{k: bad})) == D.DL_E_SHAPE, (k, bad)


def test_what_may_be_left_out():
    for call in calls(Conv):
        assert call(r=Conv.rows(bias=None)) == D.DL_E_ALIGN
    for call in calls(Ssm):
        assert call(r=Ssm.rows(skip=None, dt_bias=None, z=None, z_stride=0)) == D.DL_E_ALIGN
    for call in (Qk.forward, Qk.backward):
        assert call(r=Qk.rows(wq=None, wk=None, used=None), **({"dk": A + 4} if call == Qk.backward else {})
                    ) == D.DL_E_ALIGN
        assert call(r=Qk.rows(wq=None)) == D.DL_E_NULL        # both or neither
        assert call(d=Qk.desc(turn=0, rot=0), r=Qk.rows(pos=None, freq=None)) == D.DL_E_ALIGN


@pytest.mark.parametrize("op", [Conv, Ssm])
def test_states_and_outputs(op):
    for call in (op.step, op.prefill):
        assert call(s_out=None) == D.DL_E_NULL
        assert call(y=None) == D.DL_E_NULL
        assert call(s_in=A + 8, y=A) == D.DL_E_ALIGN
        assert call(s_out=A + 8, y=A) == D.DL_E_ALIGN
    assert op.step(s_in=None) == D.DL_E_NULL
    assert op.step(slots=A + 2, y=A) == D.DL_E_ALIGN
    assert op.prefill(s_in=None) == D.DL_E_ALIGN              # zeros: stops at the output
    assert op.backward(s_in=None) == D.DL_E_ALIGN
    assert op.backward(dy=None) == D.DL_E_NULL
    for bad in (dict(s_in=A + 8), dict(dy=A + 8), dict(ds=A + 8)):
        assert op.backward(ws=A, **bad) == D.DL_E_ALIGN
    for call in (op.prefill, op.backward):
        for field in ("cu_tokens", "seq_slot"):
            assert call(tb=tables(**{field: None})) == D.DL_E_NULL
            assert call(tb=tables(**{field: A + 2})) == D.DL_E_ALIGN
        # Nothing else of the tables is read.
        assert call(tb=tables(cu_chunks=None, chunks=None, row_slot=None, order=None)) == D.DL_E_ALIGN


@pytest.mark.parametrize("op", [Conv, Ssm, Qk])
def test_gradients(op):
    big = {Conv: ("dx", "ds"), Ssm: ("dx", "ddt", "dz", "dB", "dC", "ds"), Qk: ("dq", "dk")}[op]
    small = {Conv: ("dw", "dbias"), Ssm: ("dA", "dskip", "dbias"), Qk: ("dwq", "dwk")}[op]
    for k in big + small:
        if k != "ds":
            assert op.backward(g=op.grads(**{k: None})) == D.DL_E_NULL, k
    for k in big:
        assert op.backward(g=op.grads(**{k: A + 8}), ws=A) == D.DL_E_ALIGN, k
    for k in small:
        assert op.backward(g=op.grads(**{k: A + 2}), ws=A) == D.DL_E_ALIGN, k
    if op is not Qk:
        assert op.backward(g=op.grads(ds=None)) == D.DL_E_ALIGN
    if op is Conv:
        assert op.backward(r=op.rows(bias=None), g=op.grads(dbias=None)) == D.DL_E_ALIGN
    if op is Ssm:
        assert op.backward(r=op.rows(z=None, skip=None, dt_bias=None),
                           g=op.grads(dz=None, dskip=None, dbias=None)) == D.DL_E_ALIGN


def test_workspaces():
    for op in (Conv, Ssm, Qk):
        assert op.backward(ws=None) == D.DL_E_NULL
        assert op.backward(ws=A + 128) == D.DL_E_ALIGN
        assert op.backward(ws=A, nbytes=64) == D.DL_E_SHAPE
    assert Ssm.prefill(ws=None) == D.DL_E_NULL and Ssm.prefill(ws=A + 128, y=A) == D.DL_E_ALIGN
    assert Ssm.prefill(nbytes=64) == D.DL_E_SHAPE
    assert Ssm.prefill(tokens=10, ws=None, nbytes=0) == D.DL_E_ALIGN      # one stretch: none needed
    assert Qk.backward(r=Qk.rows(wq=None, wk=None), ws=None, nbytes=0, dk=A + 4) == D.DL_E_ALIGN
    for op in (Conv, Ssm):
        assert op.need(op.desc(), tokens=3200) > op.need(op.desc(), tokens=320) > 0
        assert op.need(op.desc(), n=0, tokens=0) == 0
        assert op.need(op.desc(), n=5) == D.DL_E_SHAPE
        assert op.need(op.desc(channels=12)) == D.DL_E_SHAPE
    assert Ssm.need(Ssm.desc(), backward=0) < Ssm.need(Ssm.desc())
    assert Ssm.need(Ssm.desc(), tokens=10, backward=0) == 0


def test_no_rows_need_no_row_pointers():
    assert Conv.prefill(r=Conv.rows(x=None, x_stride=0), y=None, tokens=0, s_out=A + 4) == D.DL_E_ALIGN
    r = Ssm.rows(x=None, dt=None, z=None, B=None, C=None, x_stride=0, dt_stride=0, z_stride=0, b_stride=0, c_stride=0)
    assert Ssm.prefill(r=r, y=None, tokens=0, s_out=A + 4) == D.DL_E_ALIGN
    assert Ssm.backward(r=r, dy=None, g=Ssm.grads(dx=None, ddt=None, dz=None, dB=None, dC=None), tokens=0) == D.DL_E_ALIGN
    assert Conv.backward(r=Conv.rows(x=None), dy=None, g=Conv.grads(dx=None), tokens=0) == D.DL_E_ALIGN


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(D.dl_conv_desc) == 6 * 4 and ctypes.sizeof(D.dl_conv_rows) == 4 * 8
    assert ctypes.sizeof(D.dl_ssm_desc) == 5 * 4 and ctypes.sizeof(D.dl_ssm_rows) == 13 * 8
    assert ctypes.sizeof(D.dl_qk_desc) == 10 * 4 and ctypes.sizeof(D.dl_qk_rows) == 9 * 8
    assert [ctypes.sizeof(t) for t in (D.dl_conv_grads, D.dl_ssm_grads, D.dl_qk_grads)] == [32, 72, 32]
