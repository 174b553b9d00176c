"""Scales whose product with log2(e) is past fp32's range are refused: a score of zero would become NaN with them."""
import os

import pytest

import paper_2606_10520_amd.unisvq as u
from test_attn_api_cpu import EINVAL, EWS, decode, prompt

pytestmark = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_past_the_range(scale):
    assert decode(width=64, ws=None, scale=scale) == EINVAL
    assert prompt(nk=1 << 20, nq=1, ws=None, scale=scale) == EINVAL


def test_scales_within_it():
    """Refused for want of a workspace only, so that nothing is launched."""
    for scale in (1e-45, 0.1, 2.3e38):
        assert decode(width=64, ws=None, scale=scale) == EWS
        assert prompt(nk=1 << 20, nq=1, ws=None, scale=scale) == EWS
