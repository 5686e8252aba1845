"""Prompts that one engine runs on several streams."""

import pytest
import torch

import sequence_reference as R

pytestmark = pytest.mark.gpu


def _engine(desc):
    from paper_2608_15533_amd import decode
    return decode.DecodeEngine(desc, 2)


def _tokens(layers):
    return [[None if x[n] is None else x[n].cuda() for n in ("q", "k", "v", "lam", "beta")]
            for x in layers]


@pytest.mark.parametrize("op", ["gdn", "kda"])
def test_two_streams_share_an_engine(op):
    """Prompts on two streams, not ordered by the program, the later calls larger than the earlier
    ones (so the workspace is replaced while one stream uses it), memory taken and written on the
    first stream in between: the bits of the same prompts one after the other."""
    from paper_2608_15533_amd import deltalog as D
    desc = D.make_desc(op, 8, 4, 64, 64, 4, "bf16")
    calls = [[40], [900, 3], [33, 700], [2500]]
    x = [[R.inputs(op, [sum(lens)], 4, 64, 64, torch.bfloat16, seed=10 * i + j) for j in range(2)]
         for i, lens in enumerate(calls)]
    tokens = [_tokens(t) for t in x]
    one = _engine(desc)
    want = [one.prefill(lens, t) for lens, t in zip(calls, tokens)]
    torch.cuda.synchronize()
    for repeat in range(3):
        two = _engine(desc)
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        got, junk = [], []
        for i, (lens, t) in enumerate(zip(calls, tokens)):
            with torch.cuda.stream(streams[i % 2]):
                got.append(two.prefill(lens, t))
            with torch.cuda.stream(streams[0]):
                junk.append(torch.empty(1 << 24, dtype=torch.uint8, device="cuda").fill_(0xff))
        for s in streams:
            s.synchronize()
        for (slots, outs), (slots_w, outs_w) in zip(got, want):
            assert slots == slots_w
            for a, b in zip(outs, outs_w):
                assert torch.equal(a, b)
        for a, b in zip(two.states, one.states):
            assert torch.equal(a.S, b.S)
