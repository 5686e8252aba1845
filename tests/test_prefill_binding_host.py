"""The binding's checks of whole-sequence calls on a host without a GPU: buffers that were made for
another descriptor or row count are refused before the library is called (the kernels would read or
write past them).  Stand-ins for device tensors: only what the checks look at."""

import types

import pytest
import torch

from paper_2608_15533_amd import deltalog as D

BF16, F32 = torch.bfloat16, torch.float32
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="stand-ins for device tensors: only on a host without a GPU")


class Device:
    """A tensor that says it is on a device."""
    is_cuda = True

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, shape

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000000


@pytest.fixture(autouse=True)
def stand_ins(monkeypatch):
    monkeypatch.setattr(torch, "zeros_like", lambda t: Device(t.dtype, *t.shape))

    def reached(*a):
        raise AssertionError("the checks let the call through")
    monkeypatch.setattr(D, "_on_current_device", reached)


def case(op="gdn", n=40, B=3, H=2, dk=64, dv=64, dtype="bf16", state="f32"):
    desc = D.make_desc(op, B, H, dk, dv, 4, dtype, state)
    it, st = D.TORCH_DTYPES[dtype], D.TORCH_DTYPES[state]
    dl = D.decay_width(desc)
    tok = D.Token(desc, n, Device(it, n, H, dk), Device(it, n, H, dk), Device(it, n, H, dv),
                  Device(F32, n, H) if dl == 1 else Device(F32, n, H, dk), Device(F32, n, H),
                  Device(F32, H, dk))
    S, o = Device(st, B, H, dk, dv), Device(it, n, H, dv)
    return desc, tok, S, o, D.Grads(desc, tok, S)


def forward(desc, tok, S, o, n=40):
    D.dl_prefill(desc, S, S, tok, o, D.ChunkTables(2, n, 3, device="cpu"), Device(torch.uint8, 1))


def backward(desc, tok, S, o, grads, n=40):
    D.dl_prefill_backward(desc, S, tok, o, None, grads, D.ChunkTables(2, n, 3, device="cpu"),
                          Device(torch.uint8, 1))


def test_what_fits_goes_through():
    desc, tok, S, o, grads = case()
    with pytest.raises(AssertionError, match="let the call through"):
        forward(desc, tok, S, o)
    with pytest.raises(AssertionError, match="let the call through"):
        backward(desc, tok, S, o, grads)
    with pytest.raises(AssertionError, match="let the call through"):
        backward(desc, tok, S, o, D.Grads(desc, tok))


@pytest.mark.parametrize("other", [dict(H=1), dict(dk=128), dict(op="kda"), dict(op="retnet")], ids=str)
def test_a_token_of_another_descriptor(other):
    desc, _, S, o, grads = case()
    tok = case(**other)[1]
    with pytest.raises(ValueError, match="token was made for another"):
        forward(desc, tok, S, o)
    with pytest.raises(ValueError, match="token was made for another"):
        backward(desc, tok, S, o, grads)


@pytest.mark.parametrize("other", [dict(n=39), dict(H=1), dict(dk=128), dict(dv=128),
                                   dict(op="kda"), dict(dtype="f32")], ids=str)
def test_gradients_of_another_call(other):
    desc, tok, S, o, _ = case()
    with pytest.raises(ValueError, match="gradients were made for another"):
        backward(desc, tok, S, o, case(**other)[4])


@pytest.mark.parametrize("other", [dict(B=2), dict(state="bf16")], ids=str)
def test_state_gradients_of_another_call(other):
    desc, tok, S, o, _ = case()
    with pytest.raises(ValueError, match="gradient of the states"):
        backward(desc, tok, S, o, case(**other)[4])


def test_rows_that_do_not_add_up():
    desc, tok, S, o, grads = case()
    with pytest.raises(ValueError, match="40 rows but the tables are for 41"):
        forward(desc, tok, S, o, n=41)
    with pytest.raises(ValueError, match="40 rows but the tables are for 41"):
        backward(desc, tok, S, o, grads, n=41)


def test_no_sequences_are_no_work(monkeypatch):
    monkeypatch.setattr(D, "_on_current_device", lambda *a: None)
    desc, tok, S, o, grads = case()
    tables = D.ChunkTables(0, 40, device="cpu")
    D.dl_chunk_tables(Device(torch.int32, 0), tables, stream=0)
    ws = types.SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, data_ptr=lambda: 0,
                               numel=lambda: 0, element_size=lambda: 1)
    D.dl_prefill(desc, S, S, tok, o, tables, ws, stream=0)
    D.dl_prefill_backward(desc, S, tok, o, None, grads, tables, ws, stream=0)
