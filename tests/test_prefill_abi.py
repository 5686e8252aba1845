"""Whole-sequence entry points on a host without a GPU: every refusal comes before any HIP call
(fake device addresses, as in test_abi_cpu.py)."""

import ctypes

import pytest
import torch

from paper_2608_15533_amd import deltalog as D

A = 0x10000000
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: only on a host without a GPU")
N = 100


def desc(_op="gdn", **kw):
    d = D.make_desc(_op, 4, 2, 128, 64, 16, "bf16")
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def token(**kw):
    t = D.dl_token(A, A + 0x1000, A + 0x2000, A + 0x3000, A + 0x4000, A + 0x5000)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def tables(**kw):
    t = D.dl_tables(A + 0x10, A + 0x20, A + 0x30, A + 0x40, A + 0x50, A + 0x60)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def grads(**kw):
    g = D.dl_grads(A, A + 0x10, A + 0x20, A + 0x30, A + 0x40, A + 0x50, A + 0x60)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def need(d, backward, n=4, tokens=N):
    return D.dl_prefill_workspace_bytes(d, n, tokens, backward)


def forward(d=None, S_in=A, S_out=A, t=None, o=A + 4, tb=None, n=4, tokens=N, ws=A, nbytes=None):
    """By default everything is in order but the output's alignment."""
    d = d or desc()
    nbytes = 1 << 40 if nbytes is None else nbytes
    return D.lib.dl_prefill(ctypes.byref(d), S_in, S_out, ctypes.byref(t or token()), o,
                            ctypes.byref(tb or tables()), n, tokens, ws, nbytes, None)


def backward(d=None, S_in=A, t=None, do=A, dS=A + 8, g=None, tb=None, n=4, tokens=N, ws=A,
             nbytes=1 << 40):
    """By default everything is in order but dS_out's alignment."""
    return D.lib.dl_prefill_backward(ctypes.byref(d or desc()), S_in, ctypes.byref(t or token()),
                                     do, dS, ctypes.byref(g or grads()),
                                     ctypes.byref(tb or tables()), n, tokens, ws, nbytes, None)


def build(lens=A, slots=A, n=4, tokens=N, num_slots=4, tb=None, err=A + 2):
    """By default everything is in order but the error word's alignment."""
    return D.lib.dl_chunk_tables(lens, slots, n, tokens, num_slots,
                                 ctypes.byref(tb or tables()), err, None)


def test_valid_calls_stop_at_the_planted_alignment():
    assert forward() == D.DL_E_ALIGN
    assert backward() == D.DL_E_ALIGN
    assert build() == D.DL_E_ALIGN


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("field,value,code", [
    ("abi_version", 3, D.DL_E_VERSION), ("op", 6, D.DL_E_UNSUPPORTED), ("dk", 96, D.DL_E_UNSUPPORTED),
    ("dv", 32, D.DL_E_UNSUPPORTED), ("merge_interval", 0, D.DL_E_UNSUPPORTED),
    ("in_dtype", 2, D.DL_E_DTYPE), ("state_dtype", 2, D.DL_E_DTYPE), ("num_slots", 0, D.DL_E_SHAPE),
    ("heads", 0, D.DL_E_SHAPE), ("heads", D.DL_MAX_HEADS + 1, D.DL_E_SHAPE),
])
def test_descriptor_rejections(call, field, value, code):
    assert call(d=desc(**{field: value})) == code


@pytest.mark.parametrize("call", [forward, backward])
def test_counts(call):
    assert call(n=5) == D.DL_E_SHAPE                     # more sequences than slots
    assert call(n=-1) == D.DL_E_SHAPE
    assert call(tokens=-1) == D.DL_E_SHAPE
    assert call(d=desc(heads=60000), tokens=2 ** 31 - 1) == D.DL_E_SHAPE   # the grid
    assert call(n=0, t=D.dl_token(), tb=D.dl_tables()) == D.DL_OK          # a no-op


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("field", ["q", "k", "v", "lam", "beta"])
def test_token_rejections(call, field):
    assert call(t=token(**{field: None})) == D.DL_E_NULL
    assert call(t=token(**{field: A + 2})) == D.DL_E_ALIGN


def test_operators_take_what_they_need():
    assert forward(d=desc("linattn"), t=token(lam=None, beta=None)) == D.DL_E_ALIGN
    assert forward(d=desc("retnet"), t=token(beta=None, u=None)) == D.DL_E_ALIGN
    assert forward(d=desc("rwkv6"), t=token(beta=None, u=None)) == D.DL_E_NULL
    assert backward(d=desc("rwkv6"), g=grads(du=None)) == D.DL_E_NULL
    assert backward(d=desc("gla"), g=grads(dbeta=None, du=None)) == D.DL_E_ALIGN
    assert backward(d=desc("gla"), g=grads(dlam=None)) == D.DL_E_NULL
    assert backward(d=desc("linattn"), g=grads(dlam=None, dbeta=None, du=None)) == D.DL_E_ALIGN


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("field", ["cu_tokens", "cu_chunks", "chunks", "seq_slot", "order"])
def test_table_rejections(call, field):
    assert call(tb=tables(**{field: None})) == D.DL_E_NULL
    assert call(tb=tables(**{field: A + 2})) == D.DL_E_ALIGN
    assert build(tb=tables(**{field: None}), err=None) == D.DL_E_NULL
    assert build(tb=tables(**{field: A + 2}), err=None) == D.DL_E_ALIGN


def test_chunk_rows_need_16_bytes():
    assert build(tb=tables(chunks=A + 8), err=None) == D.DL_E_ALIGN


@pytest.mark.parametrize("backward_pass,call", [(False, forward), (True, backward)])
def test_workspace_rejections(backward_pass, call):
    d = desc()
    assert call(d=d, ws=None) == D.DL_E_NULL
    assert call(d=d, ws=A + 128) == D.DL_E_ALIGN
    assert call(d=d, nbytes=need(d, backward_pass) - 1) == D.DL_E_SHAPE
    assert call(d=d, nbytes=need(d, backward_pass)) == D.DL_E_ALIGN       # stops later


def test_state_and_output_rejections():
    assert forward(S_out=None) == D.DL_E_NULL
    assert forward(o=None) == D.DL_E_NULL
    assert forward(S_in=None) == D.DL_E_ALIGN             # a zero start: stops at the output
    assert forward(S_in=A + 8, o=A) == D.DL_E_ALIGN
    assert forward(S_out=A + 4, o=A) == D.DL_E_ALIGN
    assert backward(do=None) == D.DL_E_NULL
    assert backward(do=A + 4, dS=None) == D.DL_E_ALIGN
    for field in ("dq", "dk", "dv"):
        assert backward(g=grads(**{field: None})) == D.DL_E_NULL
        assert backward(g=grads(**{field: A + 8}), dS=None) == D.DL_E_ALIGN
    assert backward(g=grads(dS=A + 8), dS=None) == D.DL_E_ALIGN
    assert backward(g=grads(dlam=A + 2), dS=None) == D.DL_E_ALIGN


def test_no_rows_need_no_row_pointers():
    t, g = D.dl_token(u=A), grads(dq=None, dk=None, dv=None, dbeta=None, dlam=None)
    assert forward(t=t, o=None, tokens=0, S_out=A + 4) == D.DL_E_ALIGN
    assert backward(t=t, do=None, g=g, tokens=0) == D.DL_E_ALIGN
    assert build(tb=tables(row_slot=None), tokens=0) == D.DL_E_ALIGN
    assert build(tb=tables(row_slot=None)) == D.DL_E_NULL


def test_table_counts():
    assert build(n=-1) == D.DL_E_SHAPE
    assert build(tokens=-1) == D.DL_E_SHAPE
    assert build(num_slots=0) == D.DL_E_SHAPE
    assert build(slots=None, n=5) == D.DL_E_SHAPE         # identity needs n <= num_slots
    assert build(lens=None) == D.DL_E_NULL
    assert build(lens=A + 2, err=None) == D.DL_E_ALIGN
    assert build(slots=A + 1, err=None) == D.DL_E_ALIGN
    assert build(n=0, lens=None, tb=D.dl_tables()) == D.DL_OK


def test_workspace_grows_with_what_it_holds():
    d = desc()
    assert need(d, True) > need(d, False) > 0
    assert need(d, False, tokens=3200) > need(d, False, tokens=320)
    assert need(d, False, n=1, tokens=0) > 0
    assert D.dl_prefill_workspace_bytes(d, 0, 0) == 0
    with pytest.raises(D.DeltaLogError):
        D.dl_prefill_workspace_bytes(d, 5, 10)


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(D.dl_tables) == 6 * 8
    assert ctypes.sizeof(D.dl_grads) == 7 * 8
