"""Scales of attention's scores at the ends of their type, without a GPU."""
import math

import pytest

from paper_2311_09549_amd import binding as sc
from paper_2311_09549_amd.attention import Attention


def _create(scale):
    return sc.attention_create(sc.SC_BF16, 8, 2, 128, 16, scale=scale)


@pytest.mark.parametrize("scale", [1e-50, 2.0 ** -149, 2.0 ** -127, 2.4e38, 1e39, math.inf, math.nan, -1.0, -1e-50])
def test_scales_beyond_their_type(scale):
    """A scale that 32 bits do not hold, alone and over ln 2, is no scale: neither the usual one, which 0 stands for, nor infinity."""
    for create in (_create, lambda s: Attention(8, 2, 128, scale=s)):
        with pytest.raises((ValueError, sc.ScError)):
            create(scale)


@pytest.mark.parametrize("scale", [1e-37, 0.25, 2.3e38])
def test_scales_within_their_type(scale):
    assert f"softmax_j({scale:g} *" in sc.attention_describe(_create(scale))


def test_no_scale_is_the_usual_one():
    assert "softmax_j(0.0883883 *" in sc.attention_describe(_create(0.0))
    assert "softmax_j(0.0883883 *" in Attention(8, 2, 128).describe()
    with pytest.raises(ValueError):
        Attention(8, 2, 128, scale=0.0)
