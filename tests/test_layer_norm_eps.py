"""The norms' eps has to be a normal fp32 number: the hardware's reciprocal root takes smaller ones for 0, and a
head of zeros would come out as NaN.  On a host without a GPU, as in test_layer_abi.py."""

import pytest
import torch

from paper_2608_15533_amd import deltalog as D
from test_layer_abi import Qk

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: only on a host without a GPU")


@pytest.mark.parametrize("call", [Qk.forward, Qk.backward], ids=["forward", "backward"])
@pytest.mark.parametrize("norm", ["l2", "rms"])
def test_eps_below_the_normal_numbers_is_refused(call, norm):
    kind = D.NORM_IDS[norm]
    for eps in (2.0 ** -127, 1e-45):
        assert call(d=Qk.desc(norm=kind, eps=eps)) == D.DL_E_UNSUPPORTED
    assert call(d=Qk.desc(norm=kind, eps=2.0 ** -126)) == D.DL_E_ALIGN      # looked at last
    assert call(d=Qk.desc(norm=0, eps=1e-45)) == D.DL_E_ALIGN               # no norm, no eps
