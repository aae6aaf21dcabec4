"""Angles of attention's rotation, without a GPU: as many as are read."""
import pytest

from paper_2311_09549_amd import binding as sc
from paper_2311_09549_amd.attention import Attention


@pytest.mark.parametrize("angles,rotary_dim", [(1, 4), (31, 64), (2, 128)])
def test_fewer_angles_than_pairs(angles, rotary_dim):
    """The library reads rotary_dim / 2 angles: fewer are refused before it reads behind them."""
    freq = [1.0] * angles
    with pytest.raises(ValueError, match="angles"):
        sc.attention_create(sc.SC_BF16, 8, 2, 128, 16, rotary_freq=freq, rotary_dim=rotary_dim)
    with pytest.raises(ValueError):
        Attention(8, 2, 128, rotary_freq=freq, rotary_dim=rotary_dim)


@pytest.mark.parametrize("angles,rotary_dim,pairs", [(4, 4, 2), (32, None, 32), (32, 64, 32)])
def test_as_many_angles(angles, rotary_dim, pairs):
    h = sc.attention_create(sc.SC_BF16, 8, 2, 128, 16, rotary_freq=[1.0] * angles, rotary_dim=rotary_dim)
    assert f"rotates {2 * pairs} of 128" in sc.attention_describe(h)
