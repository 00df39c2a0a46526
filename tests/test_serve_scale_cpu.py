"""The largest factor of the scores: the kernel multiplies it by log2(e) first, and a product that is no
number would make every result NaN with status 0."""
import pytest

from test_serve_refusals_cpu import ATTN, SHAPE, WS, call


@pytest.mark.parametrize("scale", [3.4e38, 2.4e38, 2.3589e38, float("inf")])
def test_refused(scale):
    assert call("tree_attention_q8", list(ATTN), ATTN, scale=scale) == SHAPE


@pytest.mark.parametrize("scale", [2.358e38, 1.0, 1e-45])
def test_not_refused_for_its_scale(scale):
    # refused for another reason that is looked at later: nothing is launched
    assert call("tree_attention_q8", list(ATTN), ATTN, scale=scale, ws_bytes=0, most=1 << 20) == WS
