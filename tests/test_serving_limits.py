"""Ends of the ranges that the serving operators take, at the C entry points on the host."""
from __future__ import annotations

import pytest

from tests.test_serving_refusals import UNSUPPORTED, WORKSPACE, attend, batch


@pytest.mark.parametrize("scale", [1.001 * 2.0 ** 127, 2.5e38, 3.4e38])
def test_scales_whose_power_of_two_leaves_fp32(scale):
    """scale / ln 2 has to be a number: 0 times infinity is none."""
    assert attend(scale=scale) == UNSUPPORTED


@pytest.mark.parametrize("scale", [1e-45, 1.0, 2.0 ** 127])
def test_scales_at_the_ends_are_taken(scale):
    assert attend(b=batch(max_kv=1 << 20, max_pages=1 << 16), scale=scale, ws=None) == WORKSPACE      # refused for something else, later
