"""Ends of the ranges that the serving operators take, at the C entry points on the host."""
from __future__ import annotations

import pytest

from tests.test_serving_refusals import SHAPE, UNSUPPORTED, WORKSPACE, attend, batch, cache


@pytest.mark.parametrize("scale", [1.001 * 2.0 ** 127, 2.5e38, 3.4e38])
def test_scales_whose_power_of_two_leaves_fp32(scale):
    """scale / ln 2 has to be a number: 0 times infinity is none."""
    assert attend(scale=scale) == UNSUPPORTED


@pytest.mark.parametrize("scale", [1e-45, 1.0, 2.0 ** 127])
def test_scales_at_the_ends_are_taken(scale):
    assert attend(b=batch(max_kv=1 << 20, max_pages=1 << 16), scale=scale, ws=None) == WORKSPACE      # refused for something else, later


def test_sequences_times_heads():
    """Rows of all sequences and kv heads are numbered in 30 bits."""
    c = cache(heads=64, token_stride=64 * 128, page_stride=16 * 64 * 128)
    call = lambda n: attend(c=c, b=batch(batch=n, tokens=n, max_q=1, max_kv=1 << 20, max_pages=1 << 16), heads=64, q_stride=8192, out_stride=8192, ws=None, wsb=0)
    assert call((1 << 20) - 1) == WORKSPACE and call(1 << 20) == SHAPE
