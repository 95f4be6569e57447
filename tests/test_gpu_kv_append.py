"""Appending to the paged cache: the rotation against its formula in 64 bits and bit for bit against the same fp32 operations, codes
against the quantizer's definition, places, padding and refusals on the device."""
from __future__ import annotations

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.serving_ref import DT, UNIT, Paged

pytestmark = pytest.mark.gpu

HALVES, PAIRS = B.SASQ_ROPE_HALVES, B.SASQ_ROPE_PAIRS


def tables(rows, rot, seed=0):
    g = torch.Generator().manual_seed(seed)
    angle = torch.rand((rows, rot // 2), generator=g, dtype=torch.float64) * 6.3
    return angle.cos().float(), angle.sin().float()


def rotate(x, cos, sin, style):
    """x [T, H, D], cos and sin [T, 1, r/2], in x's precision: each product and sum by itself."""
    half = cos.shape[-1]
    y = x.clone()
    a, b = (x[..., :half], x[..., half:2 * half]) if style == HALVES else (x[..., 0:2 * half:2], x[..., 1:2 * half:2])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    if style == HALVES:
        y[..., :half], y[..., half:2 * half] = lo, hi
    else:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = lo, hi
    return y


def codes(x16, scale):
    inv = (torch.ones(()) / scale).double()[:, None]                 # fl32(1/s); the product of 16 by 24 bits is exact in 64
    return (x16.double() * inv).round().clamp(-128, 127).to(torch.int8)


class Step:
    """New tokens of a Paged cache, and what the cache has to hold after them."""

    def __init__(self, c: Paged, rot=None, style=HALVES, rows=4096, positions=None, seed=100):
        g = torch.Generator().manual_seed(seed)
        self.c, self.style = c, style
        dt = DT[c.dtype]
        self.q, self.k, self.v = c.q, torch.randn((c.T, c.kv_heads, c.dim), generator=g).to(dt), torch.randn((c.T, c.kv_heads, c.dim), generator=g).to(dt)
        rot = c.dim if rot is None else rot
        self.cos, self.sin = tables(rows, rot, seed) if rot else (None, None)
        self.positions = positions
        used = int(c.cu[-1])
        self.pos = torch.cat([torch.arange(int(n) - new, int(n)) for (new, _), n in zip(c.lens, c.kv_len)]) if used else torch.zeros(0, dtype=torch.long)
        self.seq = torch.cat([torch.full((new,), b) for b, (new, _) in enumerate(c.lens)])
        row = self.pos if positions is None else positions[:used].long()
        self.ok = (row >= 0) & (row < rows) if rot else torch.ones(used, dtype=torch.bool)
        r = row.clamp(0, rows - 1)

        def turned(x, dtype):
            x = x[:used].to(dtype)
            return rotate(x, self.cos[r][:, None].to(dtype), self.sin[r][:, None].to(dtype), style) if rot else x
        self.q64, self.q32 = turned(self.q, torch.float64), turned(self.q, torch.float32).to(dt)
        self.k64, self.k32 = turned(self.k, torch.float64), turned(self.k, torch.float32).to(dt)
        self.mag = {n: turned(x.abs().to(torch.float64), torch.float64) for n, x in (("q", self.q), ("k", self.k))}
        self.q32[~self.ok] = 0

    def expected(self):
        k, v = self.c.k.clone(), self.c.v.clone()
        kk, vv = self.k32, self.v[:len(self.pos)]
        if self.c.int8:
            kk, vv = codes(kk, self.c.k_scale), codes(vv, self.c.v_scale)
        for t in range(len(self.pos)):
            p, b = int(self.pos[t]), int(self.seq[t])
            if not self.ok[t] or p < 0 or p // self.c.page >= self.c.width:
                continue
            page = int(self.c.table[b, p // self.c.page])
            if 0 <= page < self.c.pages:
                k[page, p % self.c.page], v[page, p % self.c.page] = kk[t], vv[t]
        return k, v

    def run(self, q="out", fused=False):
        cache, batch = self.c.on_device(B)
        up = lambda t: None if t is None else t.cuda()
        qd, kd, vd = self.q.cuda(), self.k.cuda(), self.v.cuda()
        if fused:
            both = torch.cat((qd, kd, vd), 1)
            H, Hk = self.c.heads, self.c.kv_heads
            qd, kd, vd = both[:, :H], both[:, H:H + Hk], both[:, H + Hk:]
        out = {"out": torch.full_like(self.q, 9.0, device="cuda"), "in place": qd, None: None}[q]
        B.sasq_kv_append(None if q is None else qd, kd, vd, out, cache, batch, up(self.cos), up(self.sin), up(self.positions), self.style)
        torch.cuda.synchronize()
        return out, cache

    def check(self, q="out", fused=False):
        out, cache = self.run(q, fused)
        used = len(self.pos)
        if q is not None:
            got = out.cpu()
            assert torch.equal(got[:used], self.q32)
            if q == "out":
                assert bool((got[used:] == 9.0).all())               # rows of no sequence
            # the formula in 64 bits: three fp32 roundings of at most the sum of both products, then one to 16 bits
            bound = UNIT[self.c.dtype] * self.q64.abs() + 4 * 2.0 ** -24 * 2 * self.q.abs().amax().double() + 2.0 ** -25
            assert bool(((got[:used].double() - self.q64).abs() <= bound * 1.01)[self.ok].all())
        k, v = self.expected()
        assert torch.equal(cache.k.cpu(), k) and torch.equal(cache.v.cpu(), v)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("style", [HALVES, PAIRS])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (128, 16), (128, 112), (64, 64), (64, 32), (64, 48), (128, 0), (64, 0)])
def test_rotation_and_places(dim, rot, style, dtype, int8):
    lens = [(1, 0), (5, 30), (0, 4), (40, 100), (1, 63), (3, 0)]
    Step(Paged(lens, 8, 2, dim, 16, dtype, int8, seed=1, extra_rows=3), rot, style).check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (7, 7), (32, 32), (64, 8), (5, 1), (96, 8)])
@pytest.mark.parametrize("page,order", [(16, "hnd"), (64, "nhd"), (512, "hnd")])
def test_heads_pages_and_orders(heads, kv_heads, page, order):
    Step(Paged([(1, 600), (70, 10)], heads, kv_heads, 128, page, "bf16", False, order, seed=2)).check()
    Step(Paged([(1, 600), (70, 10)], heads, kv_heads, 64, page, "f16", True, order, seed=3), style=PAIRS).check()


@pytest.mark.parametrize("q", ["out", "in place", None])
@pytest.mark.parametrize("fused", [False, True])
def test_queries_in_place_or_none_and_rows_apart(q, fused):
    Step(Paged([(9, 3), (1, 44)], 12, 4, 128, 32, "f16", seed=4)).check(q, fused)


def test_many_sequences():
    Step(Paged([((i * 5) % 4, (i * 13) % 80) for i in range(700)], 4, 2, 64, 16, "f16", seed=5)).check()


@pytest.mark.parametrize("int8", [False, True])
def test_tokens_that_are_not_stored(int8):
    c = Paged([(4, 20), (30, 10), (2, 0)], 4, 2, 64, 16, "f16", int8, seed=6, stale=3.0)
    c.table[0, 1] = -1
    c.table[1, 1] = 1 << 30
    c.kv_len = torch.tensor([24, 40, 1], dtype=torch.int32)           # the last sequence's first row is before its start
    Step(c).check()


def test_positions_outside_the_table_of_pages():
    c = Paged([(5, 60)], 4, 2, 64, 16, "f16", seed=7)
    c.kv_len = torch.tensor([c.width * 16 + 3], dtype=torch.int32)
    Step(c).check()


def test_rows_of_the_rotation_table():
    c = Paged([(6, 10), (3, 0)], 4, 2, 64, 16, "bf16", seed=8)
    Step(c, rows=50, positions=torch.tensor([0, 49, 50, -1, 7, 1 << 30, 3, 3, 0], dtype=torch.int32)).check()
    Step(Paged([(20, 40), (3, 0)], 4, 2, 64, 16, "bf16", seed=9), rows=50).check()


def test_offsets_past_32_bits():
    c = Paged([(3, 300), (70, 60)], 4, 2, 128, 64, "bf16", seed=10)
    s = Step(c)
    far = (1 << 33) // (64 * 2 * 128 * 2)
    k = torch.zeros((far + c.pages, 64, 2, 128), dtype=c.k.dtype, device="cuda")
    v = torch.zeros_like(k)
    k[far:], v[far:] = c.k.cuda(), c.v.cuda()
    batch = B.KVBatch(c.cu.cuda(), c.kv_len.cuda(), torch.where(c.table >= 0, c.table + far, -1).to(torch.int32).cuda(), c.T)
    B.sasq_kv_append(None, s.k.cuda(), s.v.cuda(), None, B.KVCache(k, v), batch, s.cos.cuda(), s.sin.cuda())
    ek, ev = s.expected()
    assert torch.equal(k[far:].cpu(), ek) and torch.equal(v[far:].cpu(), ev) and not bool(k[:far].any())


def test_codes_are_those_of_the_fake_quantizer():
    c = Paged([(40, 0)], 2, 2, 64, 16, "f16", True, seed=11)
    s = Step(c, rot=0)
    _, cache = s.run(q=None)
    for h in range(2):
        x = s.v[:, h].contiguous().cuda()
        y, q = torch.empty_like(x), torch.empty(x.shape, dtype=torch.int8, device="cuda")
        B.sasq_fakequant_fwd(x, c.v_scale[h:h + 1].cuda(), y, q)
        where = torch.arange(40)
        assert torch.equal(cache.v.cpu()[c.table[0].long()[where // 16], where % 16, h], q.cpu())


def test_in_a_graph_and_on_another_stream():
    c = Paged([(1, 30), (1, 90)], 8, 2, 128, 16, "f16", seed=12)
    s = Step(c)
    cache, batch = c.on_device(B)
    q, k, v, cos, sin = (t.cuda() for t in (s.q, s.k, s.v, s.cos, s.sin))
    out = torch.zeros_like(q)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        B.sasq_kv_append(q, k, v, out, cache, batch, cos, sin)
    st.synchronize()
    assert torch.equal(out.cpu(), s.q32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sasq_kv_append(q, k, v, out, cache, batch, cos, sin)
    for step in range(4):
        c.kv_len = torch.tensor([31 - step, 91 - 3 * step], dtype=torch.int32)
        batch.kv_len.copy_(c.kv_len)
        g.replay()
        torch.cuda.synchronize()
        e = Step(c)
        assert torch.equal(out.cpu(), e.q32)
        c.k, c.v = e.expected()
        assert torch.equal(cache.k.cpu(), c.k) and torch.equal(cache.v.cpu(), c.v)
