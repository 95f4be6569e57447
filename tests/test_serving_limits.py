"""Ends of the ranges that the serving operators take, at the C entry points on the host."""
from __future__ import annotations

import pytest

from paper_2512_14481_amd import binding as B
from tests.test_serving_refusals import SHAPE, UNSUPPORTED, WORKSPACE, attend, batch, cache


@pytest.mark.parametrize("scale", [1.001 * 2.0 ** 127, 2.5e38, 3.4e38])
def test_scales_whose_power_of_two_leaves_fp32(scale):
    """scale / ln 2 has to be a number: 0 times infinity is none."""
    assert attend(scale=scale) == UNSUPPORTED


@pytest.mark.parametrize("scale", [1e-45, 1.0, 2.0 ** 127])
def test_scales_at_the_ends_are_taken(scale):
    assert attend(b=batch(max_kv=1 << 20, max_pages=1 << 16), scale=scale, ws=None) == WORKSPACE      # refused for something else, later


def test_a_smaller_step_may_need_a_larger_workspace():
    """Fewer sequences are cut into more runs: the size is asked for each step, and what was enough for a larger one is refused."""
    lib, c = B._lib(), cache(heads=8, head_stride=128, token_stride=1024, page_stride=16384)
    size = lambda b: lib.sasq_paged_attention_workspace(c, b, 64)
    step = lambda n, keys=2000: batch(batch=n, tokens=n, max_q=1, max_kv=keys, max_pages=4096)
    assert size(step(128)) == 0 < size(step(4)) and size(step(4, 512)) == 0
    assert attend(c=c, b=step(4), heads=64, q_stride=8192, out_stride=8192, wsb=size(step(4)) - 1) == WORKSPACE
    chunks = lambda n: batch(batch=2, tokens=n, max_q=n // 2, max_kv=16000, max_pages=4096)
    assert size(chunks(8192)) < size(chunks(256))


def test_sequences_times_heads():
    """Rows of all sequences and kv heads are numbered in 30 bits, workgroups in 31."""
    c = cache(heads=64, token_stride=64 * 128, page_stride=16 * 64 * 128)
    call = lambda n, keys: attend(c=c, b=batch(batch=n, tokens=n, max_q=1, max_kv=keys, max_pages=1 << 16), heads=64, q_stride=8192, out_stride=8192, ws=None, wsb=0)
    assert call((1 << 20) - 1, 4096) == WORKSPACE and call(1 << 20, 4096) == SHAPE
    assert call(1 << 15, 1 << 20) == WORKSPACE and call(1 << 17, 1 << 20) == SHAPE                 # 2^29 and 2^31 workgroups
