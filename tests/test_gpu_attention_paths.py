"""Attention over the paged cache in the forms that only certain steps take: more sequences than a wave looks over at a time, runs of more keys
than the lanes hold places of, joins whose workgroups go round."""
from __future__ import annotations

import math

import pytest

from paper_2512_14481_amd import binding as B
from tests.serving_ref import Paged, assert_attention
from tests.test_gpu_paged_attention import SCALE, check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("batch,new", [(65, 20), (130, 20), (200, 9), (64, 70), (129, 66)])
def test_tiles_of_many_sequences(batch, new, dim, int8):
    """A tile's sequence is looked for among 64 at a time, from the last on: some have no tiles, some one, some several."""
    lens = [((0, 1, new, 2 * new + 3, new - 1)[i * 7 % 5], (i * 37) % 150) for i in range(batch)]
    check(Paged(lens, 2, 1, dim, 16, "bf16" if dim == 64 else "f16", int8, seed=batch, extra_rows=3))


@pytest.mark.parametrize("lens", [[(20, 0)] + [(0, 30)] * 200, [(0, 5)] * 200 + [(20, 7)], [(1, 9)] * 100 + [(30, 40)] + [(1, 70)] * 100])
def test_one_chunk_among_many_sequences(lens):
    check(Paged(lens, 2, 1, 64, 16, "f16", seed=51))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (128, 1024)])
@pytest.mark.parametrize("new", [20, 100])
@pytest.mark.parametrize("held", [4096, 4097, 4224, 9000])
def test_runs_of_many_keys_in_tiles(held, new, dim, page, dtype, int8):
    """Each lane knows the place of every 64th tile: 4096 keys on, the places are looked up anew.  max_kv cuts these keys into one run."""
    check(Paged([(new, held - new)], 1, 1, dim, page, dtype, int8, seed=held), max_kv=64)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new", [20, 100])
def test_a_missing_page_far_into_a_run(new, int8):
    c = Paged([(new, 9000 - new)], 1, 1, 64, 16, "f16", int8, seed=52, stale=math.nan)
    for i in (0, 255, 256, 257, 300, 560):
        c.table[0, i] = -1
    check(c, max_kv=64)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("bf16", 64), ("f16", 128), ("bf16", 128)])
@pytest.mark.parametrize("lens", [[(1, 530 + 19 * i) for i in range(40)], [(1 + i % 2, 1100 - 9 * i) for i in range(30)],
                                  [(1, 40 * i) for i in range(40)] + [(40, 700)]])
def test_joins_that_go_round(lens, dtype, dim, int8):
    """More rows with runs than the join has workgroups (2048): each takes every so manieth row of a sequence and kv head."""
    c = Paged(lens, 64, 8, dim, 64, dtype, int8, seed=53)
    cache, batch = c.on_device(B, max_q=max(n for n, _ in lens), max_kv=max(n + p for n, p in lens))
    assert len(lens) * 8 * min(16, 8 * max(n for n, _ in lens)) > 2048 and B.sasq_paged_attention_workspace(cache, batch, 64) > 0
    out, lse = run(c)
    assert_attention(c, out, lse, SCALE)
