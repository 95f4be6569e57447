"""Attention over the paged cache at the limits of its contract: lengths past the table, structures with fields that do not count, values, scores
and factors near the ends of their types."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.serving_ref import Paged, assert_attention
from tests.test_gpu_paged_attention import SCALE, run

pytestmark = pytest.mark.gpu


def fill(c, b, k=None, v=None):
    """Keys (their first channel, the others 0) and values (all channels) of sequence b's positions, one number each."""
    j = torch.arange(int(c.kv_len[b]))
    at = c.table[b].long()[j // c.page], j % c.page
    if k is not None:
        c.k[at] = 0
        c.k[at[0], at[1], :, 0] = k.to(c.k.dtype)[:, None]
    if v is not None:
        c.v[at] = v.to(c.v.dtype)[:, None, None]


def queries(c, x):
    """Every query x in its first channel, 0 in the others: the score of a key is scale * x * its first channel."""
    c.q.zero_()
    c.q[..., 0] = x


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("by", [1, 3, 40, 1000, (1 << 31) - 1])
@pytest.mark.parametrize("new,width", [(1, 21), (5, 21), (70, 21), (5, 190), (70, 190)])
def test_a_length_past_the_table(new, width, by, int8):
    """New tokens stay at the positions that the length gives, though the last ones are past the table: the others see the keys up to
    theirs, those past it the whole table.  Rows, tiles, one run and several."""
    c = Paged([(new, width * 16 - new), (2, 30)], 4, 2, 64, 16, "f16", int8, seed=41, width=width)
    c.kv_len[0] = min(width * 16 + by, (1 << 31) - 1)
    for max_kv in ("given", None):
        out, lse = run(c, max_kv=max_kv)
        assert_attention(c, out, lse, SCALE)


@pytest.mark.parametrize("lens", [[(1, 300), (3, 40)], [(1, 3000), (3, 400)], [(40, 3000), (1, 900)]])
def test_factors_of_a_16_bit_cache_are_not_read(lens):
    """The structure's factors are an int8 cache's: whatever they are, a 16-bit cache gives the same, in one run of keys and in several."""
    c = Paged(lens, 8, 2, 128, 16, "f16", seed=42)
    ref, ref_lse = run(c)
    cache, batch = c.on_device(B, max_q=max(n for n, _ in lens), max_kv=max(n + p for n, p in lens))
    factors = torch.full((2,), 3.0, device="cuda")
    cache._c.k_scale = cache._c.v_scale = factors.data_ptr()
    q, out, lse = c.q.cuda(), torch.empty_like(ref), torch.empty_like(ref_lse)
    B.sasq_paged_attention(q, out, cache, batch, B.new_workspace(B.sasq_paged_attention_workspace(cache, batch, 8)), SCALE, lse=lse)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("max_kv", ["given", 64])
@pytest.mark.parametrize("new", [1, 20])
def test_many_keys_of_little_weight(new, max_kv, int8):
    """One key 17.4 above 131071 others whose weight, 2^-25.1 of its each, is 0.36 % of the row in sum.  All values are 1, and so is the output:
    off by the rounding of the large probability and of the output (2^-11 each), of the small ones (fp16 below 2^-14 has steps of 2^-24, and
    probabilities reach 2^7 at least: 2^-32 of the largest for each), and of fp32 sums (a step of the product for every 32 keys, and a sum for every
    16 of a lane's, taken as 2^-23 each)."""
    n = 1 << 17
    c = Paged([(new, n - new)], 1, 1, 64, 256, "f16", int8, seed=43)
    queries(c, 1.0)
    if int8:
        c.k_scale[:], c.v_scale[:] = 0.2, 0.01
    k = torch.zeros(n)
    k[0] = 87 if int8 else 17.4
    fill(c, 0, k, torch.full((n,), 100.0 if int8 else 1.0))
    out, _ = run(c, max_kv=max_kv, scale=1.0)
    bound = 2 * 1.01 * 2.0 ** -11 + n * 2.0 ** -32 + (n / 32 + n / 16) * 2.0 ** -23
    assert bound < 0.7 * n * math.exp(-17.4)
    assert float((out.double() - 1).abs().max()) <= bound


@pytest.mark.parametrize("q,base", [(-2.0 ** 60, 44), (2.0 ** 60, 44), (-1.0, 20), (1.0, 20)])
@pytest.mark.parametrize("new,n", [(1, 500), (1, 2800), (30, 500), (30, 2800)])
def test_scores_far_from_zero(new, n, q, base):
    """Scores from 2e30 to 1e37, or from 1e5 to 5e11, of either sign, all different: a row's output is the value of its largest, to the bit, and
    lse that score."""
    c = Paged([(new, n - new), (1, 7)], 1, 1, 64, 64, "bf16", seed=44)
    queries(c, q)
    rank = torch.randperm(n, generator=torch.Generator().manual_seed(44))
    size = (1 + (rank % 128) / 128.0) * 2.0 ** (base + rank // 128)
    fill(c, 0, size)
    out, lse = run(c)
    for i in range(new):
        p = n - new + i
        best = int((rank[:p + 1] * q).argmax())
        at = int(c.table[0, best // 64]), best % 64
        score = SCALE * q * float(size[best])
        assert torch.equal(out[i, 0].cpu(), c.v[at][0]) and abs(float(lse[i, 0]) - score) <= 2.0 ** -21 * abs(score)


@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("dtype,q,factor", [("f16", -1.0, 2.0 ** 110), ("bf16", -2.0 ** 60, 2.0 ** 50)])
def test_scores_of_codes_far_below_zero(new, dtype, q, factor):
    c = Paged([(new, 120 - new)], 1, 1, 64, 16, dtype, True, seed=45)
    queries(c, q)
    c.k_scale[:], c.v_scale[:] = factor, 0.5
    code = 1 + torch.randperm(120, generator=torch.Generator().manual_seed(45))
    fill(c, 0, code)
    out, lse = run(c)
    for i in range(new):
        best = int(code[:121 - new + i].argmin())
        score = SCALE * q * factor * int(code[best])
        value = c.v[int(c.table[0, best // 16]), best % 16, 0].float() * 0.5
        assert torch.equal(out[i, 0].cpu().float(), value.to(c.q.dtype).float()) and abs(float(lse[i, 0]) - score) <= 2.0 ** -21 * -score


@pytest.mark.parametrize("lens", [[(1, 500), (3, 40)], [(40, 20), (1, 70)]])
@pytest.mark.parametrize("query,factor,scale", [(118, -118, 0), (125, -120, -5), (-110, 110, 0), (-120, 120, 0)])
def test_queries_of_any_size(query, factor, scale, lens):
    """bf16 queries near either end of their type over an int8 cache whose factor makes up for it."""
    c = Paged(lens, 4, 2, 128, 16, "bf16", True, seed=46)
    c.q = (c.q.float() * 2.0 ** query).to(c.q.dtype)
    c.k_scale *= 2.0 ** factor
    assert bool(torch.isfinite(c.q).all()) and bool((c.k_scale != 0).all()) and bool(torch.isfinite(c.k_scale).all())
    out, lse = run(c, scale=SCALE * 2.0 ** scale)
    assert_attention(c, out, lse, SCALE * 2.0 ** scale)


@pytest.mark.parametrize("lens", [[(1, 500), (3, 40)], [(40, 20), (1, 70)]])
@pytest.mark.parametrize("dtype,query,factor,scale", [("bf16", -126, 70, 68), ("bf16", 100, -110, 10), ("bf16", -120, -5, 125)] +
                         [(dtype, *powers) for dtype in ("f16", "bf16") for powers in ((-10, 120, -110), (0, -120, 120), (10, -140, 126))])
def test_products_of_scale_factor_and_query_of_any_size(query, factor, scale, lens, dtype):
    """Scores are finite though the product of two of the three leaves fp32 at one end or the other."""
    c = Paged(lens, 4, 2, 128, 16, dtype, True, seed=46)
    c.q = (c.q.float() * 2.0 ** query).to(c.q.dtype)
    c.k_scale *= 2.0 ** factor
    factor, scale = c.k_scale, SCALE * 2.0 ** scale
    assert bool(torch.isfinite(c.q).all()) and bool((factor != 0).all()) and bool(torch.isfinite(factor).all()) and scale < 2.0 ** 127
    out, lse = run(c, scale=scale)
    assert_attention(c, out, lse, scale)


@pytest.mark.parametrize("lens", [[(1, 500), (3, 40)], [(40, 20), (1, 70)]])
def test_the_largest_scale(lens):
    c = Paged(lens, 4, 2, 128, 16, "bf16", seed=50)
    c.q = (c.q.float() * 2.0 ** -65).to(c.q.dtype)
    c.k = (c.k.float() * 2.0 ** -65).to(c.k.dtype)
    out, lse = run(c, scale=2.0 ** 127)
    assert_attention(c, out, lse, 2.0 ** 127)


@pytest.mark.parametrize("new", [1, 30])
def test_large_values_at_scores_a_little_above_the_first(new):
    """Values near 2^117, first keys of score 0, the rest of 4.84 (2^7 times the weight): the sums over probabilities of 1 at most are finite."""
    n = 256
    c = Paged([(new, n - new)], 1, 1, 64, 64, "bf16", seed=47)
    queries(c, 1.0)
    k = torch.full((n,), 4.84375)
    k[:128 if new == 1 else 64] = 0
    fill(c, 0, k, 2.0 ** 117 * (1 + torch.rand(n, generator=torch.Generator().manual_seed(47))))
    out, lse = run(c, scale=1.0)
    assert_attention(c, out, lse, 1.0)


@pytest.mark.parametrize("new,n,low", [(1, 256, 128), (30, 256, 64), (1, 3000, 1500), (30, 3000, 1500)])
def test_large_values_of_no_weight(new, n, low):
    """The first keys' scores are 180 below the others' (a weight of 2^-259) and their values 2^120: nothing of them is in the output."""
    c = Paged([(new, n - new)], 1, 1, 64, 64, "bf16", seed=48)
    queries(c, 1.0)
    k = torch.zeros(n)
    k[:low] = -180
    v = torch.randn(n, generator=torch.Generator().manual_seed(48))
    v[:low] = 2.0 ** 120
    fill(c, 0, k, v)
    out, lse = run(c, scale=1.0)
    assert_attention(c, out, lse, 1.0)


@pytest.mark.parametrize("dtype", ["bf16"])
@pytest.mark.parametrize("power", [-118, 118])
@pytest.mark.parametrize("lens", [[(1, 500), (3, 40)], [(1, 3000), (2, 1400)], [(40, 600), (1, 70)], [(40, 3000), (1, 900)]])
def test_value_factors_of_any_size(lens, power, dtype):
    """A power of two in the factors of the values is the same power of two in the output, to the bit where that is a normal number."""
    c = Paged(lens, 4, 2, 128, 16, dtype, True, seed=49)
    ref, _ = run(c)
    c.v_scale *= 2.0 ** power
    out, _ = run(c)
    want = ref.double() * 2.0 ** power
    normal = want.abs() >= 2.0 ** -126
    assert float(normal.double().mean()) > 0.9 and torch.equal(out.double()[normal], want[normal])
