"""Scales that fr_attend_kv8 refuses before anything touches a GPU."""
import pytest

import paper_2409_06941_amd as fr
from test_cache8_host import _attend


@pytest.mark.parametrize("scale", [2.0 ** 121, 2.0 ** 127, 3e38, float("inf"), float("nan"), 0.0, -2.0 ** -149])
def test_attend_refuses_scales(scale):
    # beyond 2^120: times log2 e, or with sums of small products, they leave the range of 32 bits
    assert _attend(scale=scale) == fr.FR_ERR_ARG
