"""Attention over the paged cache against its definition in 64 bits: few rows and many, lengths around the kernels' tiles and splits,
head layouts, cache types and orders, masked places of any content, rows apart, streams, graphs."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.serving_ref import DT, Paged, assert_attention

pytestmark = pytest.mark.gpu

SCALE = 0.11


def run(c, lse=True, max_q="given", max_kv="given", q=None, out=None, scale=SCALE):
    cache, batch = c.on_device(B, max_q=max(n for n, _ in c.lens) or 1 if max_q == "given" else max_q,
                               max_kv=max(n + p for n, p in c.lens) or 1 if max_kv == "given" else max_kv)
    q = c.q.cuda() if q is None else q
    out = torch.full((c.T, c.heads, c.dim), 7.0, dtype=q.dtype, device="cuda") if out is None else out
    lse_t = torch.full((c.T, c.heads), 7.0, device="cuda") if lse else None
    ws = B.new_workspace(B.sasq_paged_attention_workspace(cache, batch, c.heads))
    ws.fill_(255)                                                    # what it holds before a call must not matter
    B.sasq_paged_attention(q, out, cache, batch, ws, scale, lse=lse_t)
    torch.cuda.synchronize()
    return out, lse_t


def check(c, **kw):
    out, lse = run(c, **kw)
    assert_attention(c, out, lse, SCALE)
    used = int(c.cu[-1])
    assert bool((out[used:] == 7.0).all()) and (lse is None or bool((lse[used:] == 7.0).all()))      # rows of no sequence
    return out, lse


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 128), (16, 2, 128), (6, 2, 64), (5, 1, 128), (20, 1, 64), (40, 1, 128)])
def test_single_tokens(heads, kv_heads, dim, dtype, int8):
    lens = [(1, p) for p in (0, 1, 14, 15, 16, 30, 31, 32, 33, 62, 63, 64, 127, 128, 200, 511, 700)]
    check(Paged(lens, heads, kv_heads, dim, 16, dtype, int8, seed=1))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("page,order", [(16, "nhd"), (32, "hnd"), (64, "nhd"), (256, "hnd"), (1024, "nhd")])
def test_pages_and_orders(page, order, int8):
    check(Paged([(1, 5), (1, 16), (1, 517), (1, 300), (1, 1023)], 8, 2, 128, page, "bf16", int8, order, seed=2))
    check(Paged([(70, 5), (33, 517), (64, 0)], 8, 2, 128, page, "f16", int8, order, seed=3))


@pytest.mark.parametrize("dtype,int8", [("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 9, 16, 17, 31, 33, 64, 65, 127, 129, 257])
def test_new_tokens(n, dtype, int8):
    check(Paged([(n, 0), (n, 1), (n, 100)], 4, 2, 128, 16, dtype, int8, seed=n))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (7, 1), (12, 4), (16, 1), (8, 4), (33, 1)])
def test_head_layouts_in_chunks(heads, kv_heads, dim):
    check(Paged([(37, 41), (130, 0), (1, 260), (6, 6)], heads, kv_heads, dim, 32, "f16", seed=5))
    check(Paged([(37, 41), (130, 0), (1, 260), (6, 6)], heads, kv_heads, dim, 32, "bf16", True, seed=6))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("past", [255, 256, 1023, 2047, 2048, 2049, 4095, 4200, 6500])
def test_long_caches_are_split(past, int8):
    check(Paged([(1, past), (1, 40), (1, past // 2)], 8, 2, 128, 64, "bf16", int8, seed=past))
    check(Paged([(3, past), (2, 700)], 8, 1, 64, 16, "f16", int8, seed=past))


def test_one_very_long_sequence():
    check(Paged([(1, 40000)], 8, 1, 128, 256, "f16", True, seed=8))
    check(Paged([(2, 33333)], 2, 2, 64, 128, "bf16", seed=9))


def test_a_long_chunk_after_a_long_past():
    check(Paged([(300, 2900), (290, 0)], 4, 1, 128, 64, "bf16", seed=10))
    check(Paged([(300, 2900), (290, 0)], 2, 1, 64, 64, "f16", True, seed=11))


@pytest.mark.parametrize("int8", [False, True])
def test_chunks_beside_single_tokens_and_idle_sequences(int8):
    lens = [(1, 900), (200, 300), (0, 50), (1, 0), (0, 0), (77, 0), (2, 2500), (1, 31), (0, 700)]
    check(Paged(lens, 8, 2, 128, 16, "bf16", int8, seed=12, extra_rows=5))
    check(Paged(lens, 5, 5, 64, 64, "f16", int8, seed=13, extra_rows=70), lse=False)


def test_many_sequences():
    check(Paged([(1 + (i * 7) % 3, (i * 37) % 190) for i in range(300)], 4, 1, 64, 16, "f16", seed=14))


@pytest.mark.parametrize("lens", [[(1, 700), (1, 90)], [(150, 100), (1, 1000)], [(4, 600)]])
def test_bounds_may_be_left_to_the_shapes(lens):
    c = Paged(lens, 8, 2, 128, 16, "f16", seed=15, width=200)
    a, la = check(c)
    b, lb = check(c, max_q=None, max_kv=None)
    assert_attention(c, b, lb, SCALE)
    check(c, max_kv=100)                                             # how far work is split, not which keys count


@pytest.mark.parametrize("stale", [math.nan, math.inf, 65504.0])
@pytest.mark.parametrize("lens", [[(1, 0), (1, 20), (1, 700)], [(40, 3), (130, 250)], [(5, 40)]])
def test_stale_places_do_not_count(lens, stale):
    for dtype in ("f16", "bf16"):
        check(Paged(lens, 8, 2, 128, 64, dtype, seed=16, stale=stale))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,past,heads,kv_heads", [(5, 30, 2, 2), (40, 3, 4, 2), (150, 77, 8, 1), (33, 500, 2, 1), (3, 61, 8, 1)])
def test_a_later_key_does_not_reach_earlier_tokens(new, past, heads, kv_heads, dim, bad):
    c = Paged([(new, past), (2, 9)], heads, kv_heads, dim, 16, "bf16", seed=17)
    p = past + new // 2                                              # the key of a token in the middle of the chunk
    for t in (c.k, c.v):
        t[c.table[0, p // 16], p % 16] = bad
    out, lse = run(c)
    clean = Paged([(new, past), (2, 9)], heads, kv_heads, dim, 16, "bf16", seed=17)
    ref, ref_lse = run(clean)
    before, after = slice(0, new // 2), slice(new // 2, new)
    assert torch.equal(out[before], ref[before]) and torch.equal(lse[before], ref_lse[before])
    assert torch.equal(out[new:], ref[new:])
    assert bool(torch.isnan(out[after]).any(-1).all())               # and the tokens that see it have it


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("new,past,kv_heads", [(1, 40, 2), (40, 3, 2), (150, 77, 1)])
def test_an_infinite_value_reaches_the_tokens_that_see_it(new, past, kv_heads, bad):
    c = Paged([(new, past)], 4, kv_heads, 128, 16, "f16", seed=18)
    p = past + new // 2
    c.v[c.table[0, p // 16], p % 16, :, 5] = bad
    out, _ = run(c)
    seen = out[new // 2:, :, 5].float().cpu()
    assert bool((torch.isnan(seen) if math.isnan(bad) else seen == bad).all())
    out[:, :, 5] = 0
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("hole", [-1, -7, 1 << 30])
def test_pages_that_are_not_there(hole, int8):
    c = Paged([(1, 200), (60, 150), (4, 100), (1, 3), (40, 0)], 8, 2, 128, 16, "f16", int8, seed=19, stale=math.nan)
    for b, i in ((0, 0), (0, 5), (0, 12), (1, 0), (1, 1), (1, 9), (2, 3), (3, 0), (4, 0), (4, 1), (4, 2)):
        c.table[b, i] = hole
    out, lse = check(c)
    assert bool((out[-41:] == 0).all()) and bool((lse[-41:] == -math.inf).all())     # rows with no key at all


def test_lengths_that_do_not_fit_are_bounded():
    c = Paged([(3, 40), (2, 10), (4, 0)], 4, 2, 64, 16, "f16", seed=20)
    c.kv_len = torch.tensor([1, -5, 4], dtype=torch.int32)           # fewer keys than rows: the first rows have none
    check(c)


@pytest.mark.parametrize("max_q,lens", [(1, [(1, 3000), (2, 3000)]), (3, [(3, 3000), (4, 3000)]), (20, [(20, 3000), (1, 90), (40, 3000)])])
def test_a_sequence_of_more_tokens_than_stated_is_left_out(max_q, lens):
    c = Paged(lens, 8, 2, 128, 64, "f16", seed=31)
    cache, batch = c.on_device(B, max_q=max_q, max_kv=max(n + p for n, p in c.lens))
    need = B.sasq_paged_attention_workspace(cache, batch, c.heads)
    ws = torch.full((need + (1 << 20),), 85, dtype=torch.uint8, device="cuda")
    q = c.q.cuda()
    out = torch.full((c.T, c.heads, c.dim), 7.0, dtype=q.dtype, device="cuda")
    B.sasq_paged_attention(q, out, cache, batch, ws[:need], SCALE)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 85).all())
    last = int(c.cu[-2])
    assert bool((out[last:] == 7.0).all())
    whole, _ = run(c, lse=False)
    assert bool((whole != 7.0).any(-1).all())
    assert float((out[:last].float() - whole[:last].float()).abs().max()) <= 2 ** -8 * float(whole.float().abs().max())


def test_rows_apart():
    c = Paged([(30, 10), (1, 200), (3, 77)], 8, 2, 128, 32, "bf16", seed=21)
    wide = torch.zeros((c.T, 13, 128), dtype=DT["bf16"], device="cuda")
    wide[:, 2:10] = c.q.cuda()
    out = torch.full((c.T, 11, 128), 3.0, dtype=DT["bf16"], device="cuda")
    _, lse = run(c, q=wide[:, 2:10], out=out[:, 1:9])
    assert_attention(c, out[:, 1:9], lse, SCALE)
    assert bool((out[:, 0] == 3).all()) and bool((out[:, 9:] == 3).all())


def test_a_cache_inside_a_larger_tensor():
    c = Paged([(1, 100), (20, 30)], 8, 2, 64, 16, "f16", seed=22)
    both = torch.full((c.pages, 2, 16, 3, 64), math.nan, dtype=DT["f16"], device="cuda")
    both[:, 0, :, :2], both[:, 1, :, :2] = c.k.cuda(), c.v.cuda()
    cache = B.KVCache(both[:, 0, :, :2], both[:, 1, :, :2])
    _, batch = c.on_device(B)
    out, lse = torch.empty_like(c.q, device="cuda"), torch.empty((c.T, 8), device="cuda")
    B.sasq_paged_attention(c.q.cuda(), out, cache, batch, B.new_workspace(B.sasq_paged_attention_workspace(cache, batch, 8)), SCALE, lse=lse)
    assert_attention(c, out, lse, SCALE)


@pytest.mark.parametrize("int8", [False, True])
def test_offsets_past_32_bits(int8):
    """Pages more than 2^32 bytes into the cache."""
    c = Paged([(1, 300), (70, 60)], 4, 2, 128, 64, "f16", int8, seed=23)
    stride = 64 * 2 * 128
    far = (1 << 33) // (stride * (1 if int8 else 2))
    k = torch.zeros((far + c.pages, 64, 2, 128), dtype=c.k.dtype, device="cuda")
    v = torch.zeros_like(k)
    k[far:], v[far:] = c.k.cuda(), c.v.cuda()
    up = lambda t: None if t is None else t.cuda()
    cache = B.KVCache(k, v, up(c.k_scale), up(c.v_scale))
    batch = B.KVBatch(c.cu.cuda(), c.kv_len.cuda(), torch.where(c.table >= 0, c.table + far, -1).to(torch.int32).cuda(), c.T)
    out, lse = torch.empty_like(c.q, device="cuda"), torch.empty((c.T, 4), device="cuda")
    B.sasq_paged_attention(c.q.cuda(), out, cache, batch, B.new_workspace(B.sasq_paged_attention_workspace(cache, batch, 4)), SCALE, lse=lse)
    assert_attention(c, out, lse, SCALE)


@pytest.mark.parametrize("lens", [[(1, 3000), (1, 100)], [(130, 700), (1, 2000)]])
def test_the_same_from_run_to_run_and_on_another_stream(lens):
    c = Paged(lens, 16, 2, 128, 16, "bf16", seed=24)
    a, la = run(c)
    for _ in range(3):
        b, lb = run(c)
        assert torch.equal(a, b) and torch.equal(la, lb)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        b, lb = run(c)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_in_a_graph():
    c = Paged([(1, 1500), (1, 90), (1, 0)], 16, 2, 128, 16, "f16", seed=25)
    cache, batch = c.on_device(B, max_q=1)                           # max_kv from the table: the graph serves longer caches too
    q, out, lse = c.q.cuda(), torch.empty_like(c.q, device="cuda"), torch.empty((c.T, 16), device="cuda")
    ws = B.new_workspace(B.sasq_paged_attention_workspace(cache, batch, 16))
    B.sasq_paged_attention(q, out, cache, batch, ws, SCALE, lse=lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sasq_paged_attention(q, out, cache, batch, ws, SCALE, lse=lse)
    for step in range(4):
        c.kv_len = torch.tensor([1501 - 300 * step, 91 - step, 1], dtype=torch.int32)
        batch.kv_len.copy_(c.kv_len)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert_attention(c, out, lse, SCALE, f"replay {step}")


def test_big_scores():
    """Scores of some thousands, one key far above the others: no overflow, and the softmax is that key."""
    c = Paged([(1, 500), (40, 20)], 4, 2, 128, 16, "f16", seed=26)
    c.q *= 20
    out, lse = run(c, scale=1.0)
    assert_attention(c, out, lse, 1.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens", [[(1, 500), (3, 40)], [(40, 20), (1, 70)]])
def test_a_scale_and_a_factor_whose_product_vanishes(lens, dtype):
    """Scores of 0 in fp32: every key counts alike, and a masked one still does not."""
    c = Paged(lens, 4, 2, 128, 16, dtype, True, seed=27)
    c.k_scale.fill_(1e-30)
    out, lse = run(c, scale=1e-30)
    assert_attention(c, out, lse, 1e-30)
