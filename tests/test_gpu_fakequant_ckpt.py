"""Fake quantization with one byte an element kept for the backward: against the definition in 64 bits, and against the form that keeps x.

Tolerance of ds: its products are exact in fp32 and added in fp64, per channel four in fp32 first (and two roundings of partial sums), so it is off by at most
8 * 2^-24 of the sum of the terms' sizes, and by one rounding of its own.
"""
from __future__ import annotations

import math

import pytest
import torch

from paper_2512_14481_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def tensors(rows, cols, dtype, pc, bits, seed=0, negative=False):
    g = torch.Generator().manual_seed(seed + rows * 7 + cols)
    x = torch.randn((rows, cols), generator=g)
    x[:, torch.rand(cols, generator=g) < 0.05] *= 40
    x[torch.rand((rows, cols), generator=g) < 0.1] = 0.0
    s = (torch.rand(cols if pc else 1, generator=g) + 0.5) * 8.0 / 2 ** (bits - 1)
    if negative:
        s = torch.where(torch.arange(s.numel()) % 2 == 0, -s, s)
    x, dy = x.to(DT[dtype]), (torch.randn((rows, cols), generator=g) * 0.1).to(DT[dtype])
    # on a border: halfway between two codes, and exactly on the ends of the range
    half = 2 ** (bits - 1)
    flat, sv = x.view(-1), s.expand(rows, cols).reshape(-1) if pc else s.expand(rows * cols)
    for i, q in enumerate((0.5, -0.5, half - 1, half - 0.5, -half, -half - 0.5, half, -half - 1)):
        if i < flat.numel():
            flat[i] = (sv[i] * q).to(DT[dtype])
    return x, s, dy


def bytes_of(x, s, bits):
    half = 2 ** (bits - 1)
    p = x.double() * (1.0 / s).double()
    r = p.round()
    q = r.clamp(-half, half - 1)
    e = (q - p).float().double()
    return torch.where(r > q, 127, torch.where(r < q, -128, (252 * e).round())).to(torch.int8), q


def ds_of(kept, dy, bits, pc):
    half = 2.0 ** (bits - 1)
    v = torch.where(kept == 127, half - 1, torch.where(kept == -128, -half, kept.double() / 252))
    t = dy.double() * v
    total = (lambda a: a.sum(0)) if pc else (lambda a: a.sum().view(1))
    return total(t), 8 * 2.0 ** -24 * total(t.abs()) + 2.0 ** -24 * total(t).abs() + 1e-45


def calls(pc):
    return ((B.sasq_fakequant_fwd_pc_ckpt, B.sasq_fakequant_bwd_pc_ckpt, B.sasq_fakequant_bwd_pc_ckpt_workspace) if pc else
            (B.sasq_fakequant_fwd_ckpt, B.sasq_fakequant_bwd_ckpt, B.sasq_fakequant_bwd_ckpt_workspace))


def check_ds(ds, kept, dy, bits, pc):
    want, tol = ds_of(kept, dy, bits, pc)
    off = (ds.cpu().double() - want).abs()
    assert (off <= tol).all(), (off.max(), tol[off.argmax()])


SIZES = [(1, 1), (1, 7), (3, 8), (2, 9), (1, 1000), (17, 64), (64, 256), (100, 33), (5, 1001), (129, 520), (1000, 513), (777, 1001), (4100, 48), (300, 4096), (70, 8200)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pc", [False, True])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, pc, dtype):
    bits = (8, 4, 2, 5)[(rows + cols) % 4]
    x, s, dy = tensors(rows, cols, dtype, pc, bits, negative=cols % 3 == 0)
    fwd, bwd, need = calls(pc)
    xd, sd, dyd = x.cuda(), s.cuda(), dy.cuda()
    y, kept = torch.full_like(xd, math.nan), torch.full((rows, cols), 99, dtype=torch.int8, device="cuda")
    fwd(xd, sd, y, kept, bits)
    want, q = bytes_of(x, s, bits)
    assert torch.equal(kept.cpu(), want)
    y0 = torch.empty_like(xd)
    (B.sasq_fakequant_fwd_pc if pc else B.sasq_fakequant_fwd)(xd, sd, y0, None, bits)
    assert torch.equal(y.view(torch.int16), y0.view(torch.int16))
    dx, ds = torch.full_like(dyd, math.nan), torch.full_like(sd, math.nan)
    ws = torch.full((need(rows, cols) + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    bwd(kept, dyd, dx, ds, ws[:-16], bits)
    keep = (want != 127) & (want != -128)
    assert torch.equal(dx.cpu().view(torch.int16), torch.where(keep, dy, 0).view(torch.int16))
    check_ds(ds, want, dy, bits, pc)
    assert (ws[-16:] == 0xFF).all()
    # no dx; dy overwritten by dx: the same
    ds2 = torch.full_like(sd, math.nan)
    bwd(kept, dyd, None, ds2, ws[:-16], bits)
    assert torch.equal(ds, ds2)
    bwd(kept, dyd, dyd, ds2, ws[:-16], bits)
    assert torch.equal(ds, ds2) and torch.equal(dyd.view(torch.int16), dx.view(torch.int16))
    # x overwritten by y: the same
    kept2 = torch.empty_like(kept)
    fwd(xd, sd, xd, kept2, bits)
    assert torch.equal(kept, kept2) and torch.equal(xd.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("pc", [False, True])
def test_against_the_form_that_keeps_x(pc):
    """dx bit for bit; ds off by at most the bytes' rounding, 1/504 of each |dy| inside the range."""
    x, s, dy = tensors(640, 1024, "f16", pc, 8, seed=3)
    fwd, bwd, need = calls(pc)
    xd, sd, dyd = x.cuda(), s.cuda(), dy.cuda()
    y, kept, dx, ds = torch.empty_like(xd), torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty_like(xd), torch.empty_like(sd)
    fwd(xd, sd, y, kept)
    bwd(kept, dyd, dx, ds, B.new_workspace(need(640, 1024)))
    dx0, ds0 = torch.empty_like(xd), torch.empty_like(sd)
    ws = B.new_workspace((B.sasq_fakequant_bwd_pc_workspace if pc else B.sasq_fakequant_bwd_workspace)(640, 1024))
    (B.sasq_fakequant_bwd_pc if pc else B.sasq_fakequant_bwd)(xd, dyd, sd, dx0, ds0, ws)
    assert torch.equal(dx.view(torch.int16), dx0.view(torch.int16))
    a = dy.double().abs()
    bound = (a.sum(0) if pc else a.sum().view(1)) / 504 * 1.001
    assert ((ds.cpu().double() - ds0.cpu().double()).abs() <= bound).all()


def test_against_differences():
    """With the rounding residuals held, y is x + s e inside the range and s q outside: ds is the slope of sum dy y over s."""
    x, s, dy = tensors(64, 96, "bf16", False, 4, seed=5)
    kept, ds = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    B.sasq_fakequant_fwd_ckpt(x.cuda(), s.cuda(), torch.empty_like(x).cuda(), kept, 4)
    B.sasq_fakequant_bwd_ckpt(kept, dy.cuda(), None, ds, B.new_workspace(B.sasq_fakequant_bwd_ckpt_workspace(64, 96)), 4)
    _, q = bytes_of(x, s, 4)
    r = (x.double() * (1.0 / s).double())
    inside = r.round() == q
    loss = lambda f: (dy.double() * torch.where(inside, x.double() + f * (q - r), f * q)).sum()
    h = 0.25
    slope = (loss(s.double() + h) - loss(s.double() - h)) / (2 * h)
    assert abs(ds.item() - slope.item()) <= dy.double().abs().sum() / 504 * 1.001


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pc", [False, True])
def test_batches(pc, dtype):
    """Up to eight tensors in a launch give what single calls give; some without dx, q, k and v on one x."""
    shapes = [(100, 256)] * 3 + [(100, 264), (1, 8), (2000, 512), (33, 104), (700, 1000)]
    t = [tensors(r, c, dtype, pc, 8, seed=i) for i, (r, c) in enumerate(shapes)]
    xs = [v[0].cuda() for v in t]
    xs[1] = xs[2] = xs[0]
    ss, dys = [v[1].cuda() for v in t], [v[2].cuda() for v in t]
    fwd, bwd, need = calls(pc)
    ys, kept = [torch.empty_like(x) for x in xs], [torch.empty(x.shape, dtype=torch.int8, device="cuda") for x in xs]
    (B.sasq_fakequant_fwd_pc_ckpt_batch if pc else B.sasq_fakequant_fwd_ckpt_batch)(list(zip(xs, ss, ys, kept)))
    dxs = [torch.full_like(x, math.nan) if i != 3 else None for i, x in enumerate(xs)]
    dss = [torch.full_like(s, math.nan) for s in ss]
    items = list(zip(kept, dys, dxs, dss))
    ws = B.new_workspace((B.sasq_fakequant_bwd_pc_ckpt_batch_workspace if pc else B.sasq_fakequant_bwd_ckpt_batch_workspace)(items))
    ws.fill_(0xFF)
    (B.sasq_fakequant_bwd_pc_ckpt_batch if pc else B.sasq_fakequant_bwd_ckpt_batch)(items, ws)
    for x, s, y, k, dy, dx, ds, (r, c) in zip(xs, ss, ys, kept, dys, dxs, dss, shapes):
        y1, k1, dx1, ds1 = torch.empty_like(x), torch.empty_like(k), torch.empty_like(x), torch.empty_like(s)
        fwd(x, s, y1, k1)
        bwd(k1, dy, dx1, ds1, B.new_workspace(need(r, c)))
        assert torch.equal(y.view(torch.int16), y1.view(torch.int16)) and torch.equal(k, k1)
        assert dx is None or torch.equal(dx.view(torch.int16), dx1.view(torch.int16))
        if pc:
            assert torch.equal(ds, ds1)
        check_ds(ds, k.cpu(), dy.cpu(), 8, pc)


@pytest.mark.parametrize("pc", [False, True])
def test_captured_and_replayed(pc):
    x, s, dy = (v.cuda() for v in tensors(300, 512, "f16", pc, 8))
    fwd, bwd, need = calls(pc)
    y, kept, dx, ds = torch.empty_like(x), torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty_like(x), torch.empty_like(s)
    ws = B.new_workspace(need(300, 512))
    fwd(x, s, y, kept)
    bwd(kept, dy, dx, ds, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fwd(x, s, y, kept)
        bwd(kept, dy, dx, ds, ws)
    for seed in (1, 2, 3):
        a = tensors(300, 512, "f16", pc, 8, seed=seed)
        for dst, src in zip((x, s, dy), a):
            dst.copy_(src.cuda())
        g.replay()
        torch.cuda.synchronize()
        k1, dx1, ds1 = torch.empty_like(kept), torch.empty_like(dx), torch.empty_like(ds)
        fwd(x, s, torch.empty_like(x), k1)
        bwd(k1, dy, dx1, ds1, B.new_workspace(need(300, 512)))
        assert torch.equal(k1, kept) and torch.equal(dx1, dx) and torch.equal(ds1, ds)


def test_far_out_of_range():
    """Values whose quotient is far past fp32's whole numbers, and infinities, are clamped."""
    x = torch.tensor([[3e4, -3e4, math.inf, -math.inf, 6e4, -6e4, 1e-7, 0.0]], dtype=torch.float16)
    for f in (1e-3, 1e-20, -1e-20):
        s = torch.tensor([f])
        kept, y = torch.empty((1, 8), dtype=torch.int8, device="cuda"), torch.empty((1, 8), dtype=torch.float16, device="cuda")
        B.sasq_fakequant_fwd_ckpt(x.cuda(), s.cuda(), y, kept)
        up, down = (127, -128) if f > 0 else (-128, 127)
        assert kept[0, :6].tolist() == [up, down] * 3 and kept[0, 7] == 0
