"""Paged caches for the tests of the serving operators, and the operators' definitions in 64 bits on the host."""
from __future__ import annotations

import math

import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}           # one rounding to the type: relative to the value


class Paged:
    """A cache on the host, filled with `stale` where no sequence has a key, and its batch.  lens: (new tokens, tokens before them)."""

    def __init__(self, lens, heads, kv_heads, dim, page, dtype="f16", int8=False, order="hnd", seed=0, stale=0.0, spare=2, extra_rows=0, width=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.kv_heads, self.dim, self.page, self.dtype, self.int8, self.order = lens, heads, kv_heads, dim, page, dtype, int8, order
        new, held = [n for n, _ in lens], [n + p for n, p in lens]
        self.T = sum(new) + extra_rows
        self.cu = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        self.kv_len = torch.tensor(held, dtype=torch.int32)
        need = [-(-n // page) for n in held]
        self.pages = sum(need) + spare
        order_of = torch.randperm(self.pages, generator=g).tolist()
        self.width = width or max(max(need), 1) + 1
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        for b, n in enumerate(need):
            for i in range(n):
                self.table[b, i] = order_of.pop()
        shape = (self.pages, page, kv_heads, dim)
        self.k_scale = self.v_scale = None
        if int8:
            self.k = torch.randint(-128, 128, shape, generator=g).to(torch.int8)
            self.v = torch.randint(-128, 128, shape, generator=g).to(torch.int8)
            sign = torch.where(torch.arange(kv_heads) % 3 == 1, -1.0, 1.0)
            self.k_scale = (0.01 + 0.02 * torch.rand(kv_heads, generator=g)) * sign
            self.v_scale = (0.01 + 0.02 * torch.rand(kv_heads, generator=g)) * sign.flip(0)
        else:
            self.k, self.v = torch.full(shape, stale, dtype=DT[dtype]), torch.full(shape, stale, dtype=DT[dtype])
            for b, n in enumerate(held):
                for j in range(0, n, page):
                    e = min(page, n - j)
                    self.k[self.table[b, j // page], :e] = torch.randn((e, kv_heads, dim), generator=g).to(DT[dtype])
                    self.v[self.table[b, j // page], :e] = torch.randn((e, kv_heads, dim), generator=g).to(DT[dtype])
        self.q = (1.5 * torch.randn((self.T, heads, dim), generator=g)).to(DT[dtype])

    def on_device(self, B, max_q=None, max_kv=None):
        """KVCache and KVBatch of the binding B."""
        def put(t):
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if self.order == "hnd" else t.cuda()
        up = lambda t: None if t is None else t.cuda()
        cache = B.KVCache(put(self.k), put(self.v), up(self.k_scale), up(self.v_scale))
        return cache, B.KVBatch(self.cu.cuda(), self.kv_len.cuda(), self.table.cuda(), self.T, max_q=max_q, max_kv=max_kv)

    def keys(self, b):
        """Positions of sequence b that are there, and their keys and values in 64 bits."""
        n = max(int(self.kv_len[b]), 0)
        j = torch.arange(min(n, self.width * self.page))
        at = self.table[b].long()[j // self.page]
        j = j[(at >= 0) & (at < self.pages)]
        at = self.table[b].long()[j // self.page]
        k, v = self.k[at, j % self.page].double(), self.v[at, j % self.page].double()
        if self.int8:
            k, v = k * self.k_scale.double()[:, None], v * self.v_scale.double()[:, None]
        return j, k, v


def attention(c: Paged, scale: float):
    """(out, lse, bound of the error of out, bound of the error of lse) of the definition, rows of no sequence left at 0.

    Each probability is rounded once to 16 bits (unit u; of an int8 cache to fp16), the output once more; scores are fp32 sums of
    `dim` products and one scale (dim + 3 roundings of 2^-24 on sum |q k|), and each exponential, sum and product of the softmax adds a
    few 2^-24 more, of the keys in whatever order: n of them at most.  fp16 probabilities below 2^-14 have steps of 2^-24."""
    u, up = UNIT[c.dtype], UNIT["f16" if c.int8 else c.dtype]
    out = torch.zeros((c.T, c.heads, c.dim), dtype=torch.float64)
    lse = torch.full((c.T, c.heads), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    G = c.heads // c.kv_heads
    for b in range(len(c.lens)):
        j, k, v = c.keys(b)
        lo, hi = int(c.cu[b]), int(c.cu[b + 1])
        for i in range(lo, hi):
            p = int(c.kv_len[b]) - (hi - lo) + (i - lo)
            n = int((j <= p).sum())
            if n == 0:
                continue
            q = c.q[i].double().view(c.kv_heads, G, c.dim)
            kk, vv = k[:n].transpose(0, 1), v[:n].transpose(0, 1)                        # [Hk, n, D]
            s = (q @ kk.transpose(1, 2)) * scale                                           # [Hk, G, n]
            size = (q.abs() @ kk.abs().transpose(1, 2)).amax(-1) * scale                   # [Hk, G]
            top = s.amax(-1, keepdim=True)
            e = (s - top).exp()
            l = e.sum(-1, keepdim=True)
            prob = e / l
            o, a = prob @ vv, prob @ vv.abs()
            low = vv.abs().sum(1)[:, None] * 2.0 ** -25 if up == UNIT["f16"] else 0.0
            in_s = ((c.dim + 3) * size + 4 * s.abs().amax(-1) + 8) * 2.0 ** -24            # of one exponent, absolute
            rel = 2 * in_s[..., None] + (n + 8) * 2.0 ** -24
            out[i], lse[i] = o.reshape(c.heads, c.dim), (top + l.log())[..., 0].reshape(c.heads)
            tol[i] = ((up * 1.01 + rel) * a + low + (u * 1.01) * o.abs() + 2.0 ** -25).reshape(c.heads, c.dim)
            tol_lse[i] = (in_s + (n + 8) * 2.0 ** -24 + lse[i].view(c.kv_heads, G).abs() * 2.0 ** -22).reshape(c.heads)
    return out, lse, tol, tol_lse


def assert_attention(c: Paged, out, lse, scale, what=""):
    ref, ref_lse, tol, tol_lse = attention(c, scale)
    used = int(c.cu[-1])
    got = out.cpu().double()[:used]
    off = (got - ref[:used]).abs() - tol[:used]
    same_nan = torch.isnan(got) & torch.isnan(ref[:used])
    off = torch.where(same_nan | (got == ref[:used]), torch.zeros_like(off), off)
    assert bool((off <= 0).all()), f"{what}: {int((~(off <= 0)).sum())} of {off.numel()} off, worst by {off.max()} at {(~(off <= 0)).nonzero()[:4].tolist()}"
    if lse is not None:
        got = lse.cpu().double()[:used]
        off = (got - ref_lse[:used]).abs() - tol_lse[:used]
        off = torch.where(got == ref_lse[:used], torch.zeros_like(off), off)
        assert bool((off <= 0).all()), f"{what}: lse off by {off.max()}"
