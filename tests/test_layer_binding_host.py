"""The binding's checks of the operators around a recurrence on a host without a GPU: tensors of the wrong
type, shape, layout or device, and buffers made for other calls, are refused before the library is called.
Stand-ins for device tensors: only what the checks look at."""

import pytest
import torch

from paper_2608_15533_amd import deltalog as D

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="stand-ins for device tensors: only on a host without a GPU")
N, B = 40, 3


class Device:
    """A tensor that says it is on a device: rows of ``shape[0]``, ``row`` elements apart."""
    is_cuda = True

    def __init__(self, dtype, *shape, row=None, index=0, dense=True):
        self.dtype, self.shape, self.index = dtype, torch.Size(shape), index
        self.device = f"cuda:{index}"
        strides, w = [], 1
        for s in reversed(shape):
            strides.append(w)
            w *= s
        self._stride = list(reversed(strides))
        if row is not None:
            self._stride[0] = row
        if not dense:
            self._stride[-1] = 2

    def stride(self, i=None):
        return tuple(self._stride) if i is None else self._stride[i]

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 0x10000000

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return 1

    def __getitem__(self, i):
        return self


@pytest.fixture(autouse=True)
def stand_ins(monkeypatch):
    like = lambda t: Device(t.dtype, *t.shape)  # noqa: E731
    monkeypatch.setattr(torch, "zeros_like", like)
    monkeypatch.setattr(torch, "zeros", lambda shape, dtype=F32, device=None: Device(dtype, *shape))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def reached(*a):
        raise AssertionError("the checks let the call through")
    for name in ("dl_conv_step", "dl_conv_prefill", "dl_conv_backward", "dl_ssm_step", "dl_ssm_prefill",
                 "dl_ssm_backward", "dl_qk_norm", "dl_qk_norm_backward"):
        monkeypatch.setattr(D._lib, name, reached)
    monkeypatch.setattr(D, "_raw_stream", lambda cur: 0)


class Tables:
    def __init__(self, tokens=N, n=B):
        self.n, self.tokens, self.struct, self.err = n, tokens, D.dl_tables(), Device(I32, 1)
        self.cu_tokens = Device(I32, n + 1)


class Conv:
    def __init__(self, n=N, D_=64, W=4, slots=B, bias=True, dtype="bf16"):
        t = D.TORCH_DTYPES[dtype]
        self.n, self.desc = n, D.make_conv_desc(slots, D_, W, dtype)
        self.args = dict(x=Device(t, n, D_), w=Device(F32, D_, W), bias=Device(F32, D_) if bias else None)
        self.s, self.y = Device(t, slots, W - 1, D_), Device(t, n, D_)

    def rows(self, **kw):
        return D.ConvRows(self.desc, self.n, **{**self.args, **kw})

    def grads(self):
        return D.ConvGrads(self.desc, self.rows(), self.s)

    def step(self, rows=None, s=None, s_out=None, y=None, slots=None):
        D.dl_conv_step(self.desc, s or self.s, s_out or self.s, rows or self.rows(), y or self.y, slots=slots)

    def prefill(self, rows=None, s=None, s_out=None, y=None, tables=None, ws=None):
        D.dl_conv_prefill(self.desc, s or self.s, s_out or self.s, rows or self.rows(), y or self.y,
                          tables or Tables())

    def backward(self, rows=None, s=None, y=None, ds=None, grads=None, tables=None, ws=None):
        D.dl_conv_backward(self.desc, s or self.s, rows or self.rows(), y or self.y, ds, grads or self.grads(),
                           tables or Tables(), ws or Device(U8, 9))


class Ssm(Conv):
    def __init__(self, n=N, D_=64, S=16, slots=B, gate=True, dtype="bf16"):
        t = D.TORCH_DTYPES[dtype]
        self.n, self.desc = n, D.make_ssm_desc(slots, D_, S, dtype)
        self.args = dict(x=Device(t, n, D_), dt=Device(t, n, D_), A=Device(F32, D_, S), Bm=Device(t, n, S),
                         Cm=Device(t, n, S), skip=Device(F32, D_), dt_bias=Device(F32, D_),
                         z=Device(t, n, D_) if gate else None)
        self.s, self.y = Device(F32, slots, D_, S), Device(t, n, D_)

    def rows(self, **kw):
        return D.SsmRows(self.desc, self.n, **{**self.args, **kw})

    def grads(self):
        return D.SsmGrads(self.desc, self.rows(), self.s)

    def step(self, rows=None, s=None, s_out=None, y=None, slots=None):
        D.dl_ssm_step(self.desc, s or self.s, s_out or self.s, rows or self.rows(), y or self.y, slots=slots)

    def prefill(self, rows=None, s=None, s_out=None, y=None, tables=None, ws=None):
        D.dl_ssm_prefill(self.desc, s or self.s, s_out or self.s, rows or self.rows(), y or self.y,
                         tables or Tables(), ws or Device(U8, 9))

    def backward(self, rows=None, s=None, y=None, ds=None, grads=None, tables=None, ws=None):
        D.dl_ssm_backward(self.desc, s or self.s, rows or self.rows(), y or self.y, ds, grads or self.grads(),
                          tables or Tables(), ws or Device(U8, 9))


class Qk:
    def __init__(self, n=N, H=4, d=64, rep=2, turn="halves", dtype="bf16", weight=True):
        t = D.TORCH_DTYPES[dtype]
        self.n, self.desc = n, D.make_qk_desc(H, d, "rms", turn, None, rep, dtype)
        self.args = dict(q=Device(t, n, H, d), k=Device(t, n, H, d), pos=Device(I32, n), freq=Device(F32, d // 2),
                         wq=Device(F32, d) if weight else None, wk=Device(F32, d) if weight else None)
        self.out = Device(t, n, H * rep, d)

    def rows(self, **kw):
        return D.QkRows(self.desc, self.n, **{**self.args, **kw})

    def grads(self):
        return D.QkGrads(self.desc, self.rows())

    def forward(self, rows=None, q=None, k=None):
        D.dl_qk_norm(self.desc, rows or self.rows(), q or self.out, k or self.out)

    def backward(self, rows=None, q=None, k=None, grads=None, ws=None):
        D.dl_qk_norm_backward(self.desc, rows or self.rows(), q or self.out, k or self.out,
                              grads or self.grads(), ws or Device(U8, 9))


ALL = [(c, f) for c in (Conv, Ssm) for f in ("step", "prefill", "backward")] + [(Qk, "forward"), (Qk, "backward")]
every = pytest.mark.parametrize("case,call", ALL, ids=[f"{c.__name__}-{f}" for c, f in ALL])
packed = pytest.mark.parametrize("case,call", [a for a in ALL if a[0] is not Qk and a[1] != "step"], ids=str)


def made(case, call, **kw):
    return case(**({"n": B} if call == "step" else {}), **kw)


@every
def test_what_fits_goes_through(case, call):
    with pytest.raises(AssertionError, match="let the call through"):
        getattr(made(case, call), call)()


@every
def test_rows_of_another_descriptor(case, call):
    c = made(case, call)
    others = {Conv: [dict(D_=72), dict(W=3), dict(dtype="f32")], Ssm: [dict(D_=72), dict(S=32), dict(dtype="f32")],
              Qk: [dict(H=2), dict(d=128), dict(rep=1), dict(turn="pairs"), dict(dtype="f32")]}[case]
    for other in others:
        with pytest.raises(ValueError, match="rows were made for another"):
            getattr(c, call)(rows=made(case, call, **other).rows())
    if case is not Qk:                                      # rows do not depend on the slots
        with pytest.raises(AssertionError, match="let the call through"):
            getattr(c, call)(rows=made(case, call, slots=B + 1).rows())


@pytest.mark.parametrize("case", [Conv, Ssm, Qk])
def test_gradients_of_another_call(case):
    c = case()
    others = {Conv: [dict(D_=72), dict(n=39), dict(bias=False)], Ssm: [dict(S=32), dict(n=39), dict(gate=False)],
              Qk: [dict(H=2), dict(n=39), dict(weight=False)]}[case]
    for other in others:
        with pytest.raises(ValueError, match="gradients were made for other"):
            c.backward(grads=case(**other).grads())
    if case is not Qk:
        with pytest.raises(ValueError, match="gradient of the states"):
            c.backward(grads=case(slots=B + 1).grads())


@packed
def test_rows_that_do_not_add_up(case, call):
    with pytest.raises(ValueError, match="40 rows but the tables are for 41"):
        getattr(case(), call)(tables=Tables(41))


def test_norm_tables():
    with pytest.raises(ValueError, match="40 rows but the tables are for 41"):
        Qk().rows(tables=Tables(41))
    Qk().rows(tables=Tables())


@pytest.mark.parametrize("case", [Conv, Ssm, Qk])
def test_layouts(case):
    c = case()
    for name, t in c.args.items():
        if t is None:
            continue
        other = F32 if t.dtype != F32 else BF16
        for bad in (Device(other, *t.shape), Device(t.dtype, *t.shape, 1), Device(t.dtype, t.shape[0] + 1, *t.shape[1:])):
            with pytest.raises(ValueError, match=name):
                c.rows(**{name: bad})
        with pytest.raises(ValueError, match="tensors on cuda"):
            c.rows(**{name: Device(t.dtype, *t.shape, index=1)})
    wide = {Conv: ("x",), Ssm: ("x", "dt", "Bm", "Cm", "z"), Qk: ("q", "k")}[case]
    for name in wide:
        t = c.args[name]
        width = t.shape.numel() // N
        c.rows(**{name: Device(t.dtype, *t.shape, row=width + 8)})
        for row in (width - 8, width + 4, 0):
            with pytest.raises(ValueError, match=f"{name}: rows"):
                c.rows(**{name: Device(t.dtype, *t.shape, row=row)})
        with pytest.raises(ValueError, match=f"{name}: a row must be dense"):
            c.rows(**{name: Device(t.dtype, *t.shape, dense=False)})
    needed = {Conv: ("x", "w"), Ssm: ("x", "dt", "A", "Bm", "Cm"), Qk: ("q", "k", "pos", "freq")}[case]
    for name in needed:
        with pytest.raises(ValueError, match=f"{name} is required"):
            c.rows(**{name: None})
    if case is Qk:
        with pytest.raises(ValueError, match="both"):
            c.rows(wk=None)


@every
def test_states_outputs_and_workspaces(case, call):
    c = made(case, call)
    if case is Qk:
        for name in ("q", "k"):
            for bad in (Device(F32, *c.out.shape), Device(BF16, N, 4, 64)):
                with pytest.raises(ValueError, match=name):
                    getattr(c, call)(**{name: bad})
    else:
        for bad in (Device(F32, *c.y.shape), Device(BF16, c.n + 1, 64)):
            with pytest.raises(ValueError, match="y"):
                getattr(c, call)(y=bad)
        for bad in (Device(U8, *c.s.shape), Device(c.s.dtype, B + 1, *c.s.shape[1:])):
            with pytest.raises(ValueError, match="_in"):
                getattr(c, call)(s=bad)
        with pytest.raises(ValueError, match="the current device is"):
            getattr(c, call)(s=Device(c.s.dtype, *c.s.shape, index=1))
    if call == "backward" or (case is Ssm and call == "prefill"):
        host = Device(U8, 9)
        host.is_cuda = False
        with pytest.raises(ValueError, match="workspace"):
            getattr(c, call)(ws=host)


def test_tensors_of_another_device():
    c = Conv(n=B)
    for t in c.args.values():
        t.index = 1
    with pytest.raises(ValueError, match="current device is cuda:0"):
        c.step()


def test_a_descriptor_that_changed():
    c = Conv(n=B)
    rows = c.rows()
    c.desc.width = 3
    with pytest.raises(ValueError, match="rows were made for another"):
        c.step(rows=rows)
