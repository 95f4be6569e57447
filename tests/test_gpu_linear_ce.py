"""Cross entropy of a frozen head against its definition in 64 bits: sizes, masks, strides, weights, pieces, graphs."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.ce_ref import DT, Head, check

pytestmark = pytest.mark.gpu


def heads(w, grad=True):
    w = w.cuda()
    V, H = w.shape
    made = []
    for form in (B.SASQ_HEAD_LOGITS, B.SASQ_HEAD_GRAD):
        h = torch.full((B.sasq_head_bytes(V, H, form),), 0xFF, dtype=torch.uint8, device="cuda")
        B.sasq_prepare_head(w, h, form)
        made.append(h)
    return made


def call(p, piece=0, grad=True, lse=True, mean=True, row_weight=None, scale=1.0, x=None, dx=None, hw=None):
    hl, hg = hw or heads(p.w)
    x = p.x.cuda() if x is None else x
    nan = lambda n: torch.full((n,), math.nan, device="cuda")
    out = {"loss": nan(p.T), "lse": nan(p.T) if lse else None, "mean": nan(1) if mean else None,
           "dx": (torch.full((p.T, p.H), math.nan, dtype=DT[p.dtype], device="cuda") if dx is None else dx) if grad else None}
    need = B.sasq_linear_ce_workspace(p.T, p.V, p.H, grad, piece)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN wherever nothing was written
    B.sasq_linear_ce(x, hl, p.t.cuda(), out["loss"], p.V, ws[:need], lse=out["lse"], mean=out["mean"], dx=out["dx"],
                     head_grad=hg if grad else None, row_weight=None if row_weight is None else row_weight.cuda(), scale=scale, piece=piece)
    torch.cuda.synchronize()
    assert (ws[need:] == 0xFF).all()
    return out


SIZES = [(1, 1, 1), (1, 7, 64), (3, 257, 8), (2, 2, 3), (5, 1000, 100), (16, 1000, 256), (17, 513, 72), (64, 1000, 256), (65, 2050, 192), (130, 513, 65), (257, 2049, 320),
         (300, 5000, 640), (1, 5003, 1000)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H", SIZES)
def test_sizes(T, V, H, dtype):
    p = Head(T, V, H, dtype, seed=T + V)
    scale = 64.0
    check(call(p, scale=scale), p.reference(scale=scale))


@pytest.mark.parametrize("dtype,left_out,grad", [("f16", 0.0, True), ("bf16", 0.55, True), ("f16", 0.2, False)])
@pytest.mark.parametrize("T,V,H", [(520, 9000, 4096), (1100, 16001, 4096), (2100, 9000, 2048), (129, 33000, 1024), (3000, 24000, 320)])
def test_large_tiles(T, V, H, dtype, left_out, grad):
    """256x256 tiles, whole rounds and last rounds as halves, by the rows that count; contractions cut into parts; several pieces (the definition on the device)."""
    p = Head(T, V, H, dtype, seed=T, left_out=left_out)
    check(call(p, grad=grad, scale=256.0), p.reference(scale=256.0, device="cuda"))


@pytest.mark.parametrize("dtype,left_out,grad", [("f16", 0.0, True), ("bf16", 0.3, True), ("f16", 0.3, False)])
@pytest.mark.parametrize("T,V,H", [(1, 300, 4097), (2, 4096, 2050), (3, 8300, 4096), (16, 8192, 2049), (17, 300, 2048), (20, 4097, 2100), (33, 2049, 2113), (64, 4096, 2056),
                                   (64, 8191, 2050), (64, 8200, 2048)])
def test_few_rows_of_long_ones(T, V, H, dtype, left_out, grad):
    """At most 64 rows, long enough that the logits' workgroups take 16, 32 or 64 columns by the vocabulary's size."""
    p = Head(T, V, H, dtype, seed=T + V, left_out=left_out)
    check(call(p, grad=grad, scale=32.0), p.reference(scale=32.0, device="cuda"))


@pytest.mark.parametrize("dtype,left_out,grad", [("f16", 0.0, True), ("bf16", 0.4, True), ("f16", 0.4, False)])
@pytest.mark.parametrize("T,V,H", [(65, 600, 104), (100, 8192, 512), (128, 8200, 64), (193, 1000, 2048), (500, 513, 2056), (1000, 700, 256), (2048, 65, 72), (2049, 65, 72)])
def test_many_rows_of_small_heads(T, V, H, dtype, left_out, grad):
    """Up to 2048 rows go by 64 a workgroup where the head is small; limits of that."""
    p = Head(T, V, H, dtype, seed=T + V, left_out=left_out)
    check(call(p, grad=grad, scale=32.0), p.reference(scale=32.0, device="cuda"))


@pytest.mark.parametrize("dtype,left_out,grad", [("f16", 0.0, True), ("bf16", 0.4, True), ("f16", 0.4, False)])
@pytest.mark.parametrize("T,V,H", [(130, 8209, 65), (300, 8193, 333), (70, 9001, 1), (2100, 513, 65), (65, 8193, 8), (257, 8449, 2049)])
def test_tiles_of_odd_sizes(T, V, H, dtype, left_out, grad):
    p = Head(T, V, H, dtype, seed=T + H, left_out=left_out)
    check(call(p, grad=grad, scale=32.0), p.reference(scale=32.0, device="cuda"))


@pytest.mark.parametrize("T,V", [(300, 700), (300, 8300)])
def test_many_rows_apart_weighted_and_in_place(T, V):
    """Strides, weights, a scale, the gradient in place of x: 64 rows a workgroup, and tiles."""
    p = Head(T, V, 72, "bf16", seed=1, left_out=0.2)
    rw = torch.randn(T, generator=torch.Generator().manual_seed(8))
    ref = p.reference(row_weight=rw, scale=-3.0, device="cuda")
    hw = heads(p.w)
    for pad in (8, 3):
        x = torch.full((T, 72 + pad), 7.0, dtype=DT["bf16"], device="cuda")
        x[:, :72] = p.x.cuda()
        check(call(p, hw=hw, x=x[:, :72], row_weight=rw, scale=-3.0), ref)
        check(call(p, hw=hw, x=x[:, :72], dx=x[:, :72], row_weight=rw, scale=-3.0), ref)
        assert (x[:, 72:] == 7.0).all()


@pytest.mark.parametrize("T,V", [(130, 700), (150, 8300)])
def test_many_rows_captured(T, V):
    """Replayed with other rows left out, as many as none: what eager calls give."""
    a, b, c = (Head(T, V, 96, "f16", seed=20 + i, left_out=o) for i, o in enumerate((0.3, 0.9, 1.0)))
    hl, hg = heads(a.w)
    x, t = a.x.cuda(), a.t.cuda()
    ws = B.new_workspace(B.sasq_linear_ce_workspace(T, V, 96, True))
    loss, lse, mean, dx = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(x)
    run = lambda: B.sasq_linear_ce(x, hl, t, loss, V, ws, lse=lse, mean=mean, dx=dx, head_grad=hg)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for p in (b, a, c, b, a):
        x.copy_(p.x.cuda())
        t.copy_(p.t.cuda())
        g.replay()
        torch.cuda.synchronize()
        want = call(p, hw=(hl, hg))
        for got, k in ((loss, "loss"), (lse, "lse"), (mean, "mean"), (dx, "dx")):
            assert torch.equal(got, want[k]), k


@pytest.mark.parametrize("T,V", [(300, 8300), (300, 600)])
def test_many_rows_of_which_one_is_not_finite(T, V):
    p = Head(T, V, 64, "f16", seed=43)
    ref = p.reference(row_weight=torch.ones(T))
    p.x = p.x.clone()
    p.x[3, 5], p.x[257, 0] = math.nan, math.inf
    out = call(p, row_weight=torch.ones(T))
    ok = torch.ones(T, dtype=torch.bool)
    ok[3] = ok[257] = False
    for k in ("loss", "lse", "dx"):
        v, (want, tol) = out[k].cpu().double(), ref[k]
        assert ((v - want).abs() <= tol)[ok].all() and not torch.isfinite(v[~ok]).all(), k


@pytest.mark.parametrize("T,V,H", [(4093, 300, 64), (8191, 300, 64), (8193, 300, 64), (9001, 130, 100), (20000, 65, 72)])
def test_many_rows_packed(T, V, H):
    """The rows that count are packed by the kernel that stages them, or, where they are many, by one of its own."""
    p = Head(T, V, H, "bf16", seed=T, left_out=0.4)
    check(call(p, scale=64.0), p.reference(scale=64.0, device="cuda"))


@pytest.mark.parametrize("T,V,H", [(384, 30000, 1024), (640, 9000, 2048), (257, 33000, 520), (1281, 16000, 512)])
def test_a_last_row_of_tiles_that_is_half_full(T, V, H):
    p = Head(T, V, H, "f16", seed=T)
    check(call(p, scale=64.0), p.reference(scale=64.0, device="cuda"))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H", [(1, 1, 1), (16, 1000, 256), (50, 700, 64), (300, 5000, 640)])
def test_without_gradient(T, V, H, dtype):
    p = Head(T, V, H, dtype, seed=3, left_out=0.2)
    check(call(p, grad=False), p.reference())
    check(call(p, grad=False, lse=False, mean=False), p.reference())


@pytest.mark.parametrize("left_out", [0.3, 0.95, 1.0])
@pytest.mark.parametrize("T,V,H", [(1, 300, 64), (40, 300, 100), (700, 1030, 128), (2500, 300, 64)])
def test_left_out_rows(T, V, H, left_out):
    """Left-out rows are 0 whatever they hold; the others do not see them."""
    p = Head(T, V, H, "bf16", seed=5, left_out=left_out)
    ref = p.reference()
    out = (p.t < 0) | (p.t >= V)
    p.x[out] = math.nan
    p.x[out & (torch.arange(T) % 3 == 0)] = math.inf
    check(call(p), ref)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H,piece", [(7, 3000, 128, 256), (7, 3000, 128, 1024), (300, 1500, 200, 256), (300, 2817, 192, 512), (600, 2561, 640, 2560), (20, 1000, 64, 4096)])
def test_pieces(T, V, H, piece, dtype):
    """Each piece may raise a row's maximum or not; the last may hold a single column."""
    p = Head(T, V, H, dtype, seed=11, left_out=0.1)
    check(call(p, piece=piece, scale=32.0), p.reference(scale=32.0))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("order", ["up", "down"])
def test_pieces_with_steep_maxima(dtype, order):
    """Logits over a range of 120, ascending or descending from piece to piece: sums of earlier pieces vanish, or those of later ones."""
    p = Head(40, 1500, 64, dtype, seed=2, sure=0.0)
    ramp = torch.linspace(-60, 60, 1500)
    p.x[:, 0] = 1.0
    p.w[:, 0] = (ramp if order == "up" else ramp.flip(0)).to(DT[dtype])
    check(call(p, piece=256), p.reference())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_sure_rows(dtype):
    """Targets that are all but certain: losses down to 1e-7 and less, and gradients as small; also targets all but excluded."""
    p = Head(64, 600, 128, dtype, seed=9, sure=0.0)
    size = torch.linspace(-12, 26, 64)
    x = torch.randn((64, 128), generator=torch.Generator().manual_seed(4)) * 0.3
    w = p.w.float()
    p.x = (x + size[:, None] * w[p.t.long()] / (w[p.t.long()] ** 2).sum(1, keepdim=True)).to(DT[dtype])
    ref = p.reference(scale=2.0 ** 14)
    assert ref["loss"][0].min() < 1e-7 and ref["loss"][0].max() > 10
    check(call(p, scale=2.0 ** 14), ref)


def test_row_weights_and_scale():
    p = Head(90, 700, 96, "bf16", seed=1, left_out=0.2)
    rw = torch.randn(90, generator=torch.Generator().manual_seed(8))
    rw[3] = 0.0
    check(call(p, row_weight=rw, scale=-3.0), p.reference(row_weight=rw, scale=-3.0))


@pytest.mark.parametrize("x_pad,dx_pad,H", [(8, 16, 64), (3, 0, 64), (0, 5, 64), (64, 64, 100), (1, 1, 33)])
def test_rows_apart(x_pad, dx_pad, H):
    p = Head(50, 400, H, "f16", seed=6)
    x = torch.full((50, H + x_pad), math.nan, dtype=DT["f16"], device="cuda")
    x[:, :H] = p.x.cuda()
    dx = torch.full((50, H + dx_pad), 7.0, dtype=DT["f16"], device="cuda")
    check(call(p, x=x[:, :H], dx=dx[:, :H]), p.reference())
    assert (dx[:, H:] == 7.0).all()
    w = torch.full((400, H + x_pad), math.nan, dtype=DT["f16"], device="cuda")
    w[:, :H] = p.w.cuda()
    for a, b in zip(heads(p.w), heads(w[:, :H])):
        assert torch.equal(a, b)


def test_gradient_in_place_of_x():
    p = Head(70, 900, 128, "bf16", seed=7, left_out=0.2)
    apart = call(p)
    x = p.x.cuda()
    same = call(p, x=x, dx=x)
    for k in apart:
        assert torch.equal(apart[k], same[k]), k


@pytest.mark.parametrize("V,H", [(1, 1), (40, 33), (130, 64), (1000, 200)])
def test_layouts(V, H):
    """Both layouts element by element; places past the matrix, up to 64 columns, hold zeros."""
    w = torch.randn((V, H), generator=torch.Generator().manual_seed(V)).to(torch.float16)
    up = lambda n, m: -(-n // m) * m
    for got, rows, cols, m in zip(heads(w), (V, H), (H, V), (w, w.t())):
        R, C = up(rows, 16), up(cols, 64)
        kt = C // 32 | 1                                                        # an odd number of blocks a row of them
        assert got.numel() == R * kt * 64
        full = torch.zeros((R, C), dtype=torch.float16)
        full[:rows, :cols] = m
        r, c = torch.arange(R)[:, None], torch.arange(C)[None]
        swz = ((r >> 1) & 3) ^ ((r >> 3) & 1)
        at = ((r // 16) * kt + c // 32) * 512 + ((4 * (r % 16) + (((c >> 3) & 3) ^ swz)) << 3) + (c & 7)
        assert torch.equal(got.cpu().view(torch.float16)[at], full)


def test_same_from_run_to_run():
    p = Head(333, 5003, 200, "f16", seed=12, left_out=0.1)
    hw = heads(p.w)
    first = call(p, hw=hw)
    for _ in range(3):
        again = call(p, hw=hw)
        for k in first:
            assert torch.equal(first[k], again[k]), k


def test_differences():
    """dx against differences of the loss itself, in the direction of dx and in a random one."""
    p = Head(4, 300, 64, "f16", seed=13, sure=4.0)
    hw = heads(p.w)
    got = call(p, hw=hw, row_weight=torch.ones(4))
    base = p.x.double()
    for direction in (got["dx"].cpu().double(), torch.randn((4, 64), generator=torch.Generator().manual_seed(1)).double()):
        step = 0.25 * direction / direction.norm(dim=1, keepdim=True)
        ends = []
        for sign in (1, -1):
            q = Head(4, 300, 64, "f16", seed=13, sure=4.0)
            q.x = (base + sign * step).to(torch.float16)
            ends.append((q.x.double(), call(q, hw=hw, grad=False)["loss"].cpu().double()))
        moved = ends[0][0] - ends[1][0]
        slope = (got["dx"].cpu().double() * moved).sum(1)
        # third-order term of the central difference: the third derivative along a unit direction is at most 2 max|W_v - W_t|^3, times (step^3) / 24 * 2
        third = 2 * (2 * p.w.double().norm(dim=1).max()) ** 3 * (0.26 ** 3) / 12
        assert ((ends[0][1] - ends[1][1]) - slope).abs().max() < third + 0.51 * 2.0 ** -9


def test_captured_and_replayed():
    """A graph of two calls, replayed with new inputs between, gives what eager calls on a workspace of their own give."""
    a, b = Head(37, 700, 96, "bf16", seed=20, left_out=0.3), Head(37, 700, 96, "bf16", seed=21, left_out=0.6)
    b.w = a.w
    hl, hg = heads(a.w)
    x, t = a.x.cuda(), a.t.cuda()
    ws = B.new_workspace(B.sasq_linear_ce_workspace(37, 700, 96, True))
    loss, lse, mean = torch.empty(37, device="cuda"), torch.empty(37, device="cuda"), torch.empty(1, device="cuda")
    dx = torch.empty_like(x)
    run = lambda: B.sasq_linear_ce(x, hl, t, loss, 700, ws, lse=lse, mean=mean, dx=dx, head_grad=hg)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
        run()
    for p in (a, b, a, b):
        x.copy_(p.x.cuda())
        t.copy_(p.t.cuda())
        g.replay()
        torch.cuda.synchronize()
        want = call(p, hw=(hl, hg))
        for got, k in ((loss, "loss"), (lse, "lse"), (mean, "mean"), (dx, "dx")):
            assert torch.equal(got, want[k]), k


@pytest.mark.parametrize("T,V,H,piece", [(30, 700, 64, 0), (30, 700, 64, 256), (200, 700, 64, 0), (200, 900, 64, 512)])
def test_no_row_counts(T, V, H, piece):
    """All rows left out, in each form, and then a call whose rows count on the same workspace."""
    p = Head(T, V, H, "f16", seed=40)
    hw = heads(p.w)
    ws = B.new_workspace(max(B.sasq_linear_ce_workspace(T, V, H, g, piece) for g in (False, True)))
    ws.fill_(0xFF)
    t = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    for targets in (t, p.t.cuda(), t):
        for dx in (None, torch.full((T, H), 5.0, dtype=torch.float16, device="cuda")):
            loss, lse, mean = (torch.full((n,), 5.0, device="cuda") for n in (T, T, 1))
            B.sasq_linear_ce(p.x.cuda(), hw[0], targets, loss, V, ws, lse=lse, mean=mean, dx=dx, head_grad=hw[1], piece=piece)
            out = {"loss": loss, "lse": lse, "mean": mean, "dx": dx}
            if targets is t:
                assert all(v is None or not v.any() for v in out.values())
            else:
                check(out, p.reference())


def test_two_graphs_on_one_workspace():
    """Graphs of two sizes that share a workspace, replayed in turn."""
    a, b = Head(20, 700, 64, "f16", seed=41), Head(150, 700, 64, "f16", seed=42)
    b.w = a.w
    hw = heads(a.w)
    ws = B.new_workspace(max(B.sasq_linear_ce_workspace(n, 700, 64, True) for n in (20, 150)))
    graphs = []
    for p in (a, b):
        x, t, loss, mean, dx = p.x.cuda(), p.t.cuda(), torch.empty(p.T, device="cuda"), torch.empty(1, device="cuda"), torch.empty(p.T, 64, dtype=torch.float16, device="cuda")
        run = lambda x=x, t=t, loss=loss, mean=mean, dx=dx: B.sasq_linear_ce(x, hw[0], t, loss, 700, ws, mean=mean, dx=dx, head_grad=hw[1])
        run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        graphs.append((g, {"loss": loss, "mean": mean, "dx": dx}, p.reference(), x))
    for _ in range(3):
        for g, out, ref, _x in graphs:
            for v in out.values():
                v.fill_(math.nan)
            g.replay()
            torch.cuda.synchronize()
            check(out, ref)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_row_that_is_not_finite(dtype):
    """A NaN or an infinity in a counted row's x stays in that row (and in the mean)."""
    for T in (20, 90):
        p = Head(T, 600, 64, dtype, seed=43)
        ref = p.reference(row_weight=torch.ones(T))
        x = p.x.clone()
        x[3, 5], x[11, 0] = math.nan, math.inf
        p.x = x
        out = call(p, row_weight=torch.ones(T))
        ok = torch.ones(T, dtype=torch.bool)
        ok[3] = ok[11] = False
        assert not torch.isfinite(out["loss"][3]) and not torch.isfinite(out["mean"]).any()
        for k in ("loss", "lse", "dx"):
            v, (want, tol) = out[k].cpu().double(), ref[k]
            assert ((v - want).abs() <= tol)[ok].all(), k


@pytest.mark.parametrize("T,V,piece", [(20, 65, 0), (20, 257, 256), (100, 257, 0), (100, 129, 0)])
def test_low_logits_and_a_group_of_the_target_alone(T, V, piece):
    """All logits about -150, and the target alone behind the last whole group of columns: it is in no sum, and its group has no maximum of its own."""
    p = Head(T, V, 64, "bf16", seed=46, sure=0.0)
    p.w = (p.w.float() - 150.0 / 64).to(torch.bfloat16)
    p.x = (1.0 + 0.05 * p.x.float()).to(torch.bfloat16)
    p.t[::2] = V - 1
    assert p.reference()["lse"][0].max() < -100
    check(call(p, piece=piece), p.reference())


@pytest.mark.parametrize("T,V", [(40, 300), (130, 300)])
def test_equal_logits_and_one_column(T, V):
    """Zero heads: all logits equal, loss ln V; a vocabulary of one entry: loss 0 and no gradient."""
    p = Head(T, V, 64, "bf16", seed=44)
    p.w = torch.zeros_like(p.w)
    check(call(p), p.reference())
    q = Head(T, 1, 64, "bf16", seed=45)
    out = call(q)
    assert not out["loss"].any() and not out["dx"].any()


def test_a_long_vocabulary_and_row():
    """Offsets past 2^31 bytes in the head's layouts: entries and channels at the far end are those of a small head that holds them alone."""
    V, H, T = 300000, 4096, 3                                     # 2.4 GB a layout
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    part = torch.randn((1000, H), generator=g, device="cuda").mul_(1 / 64).to(torch.bfloat16)
    w[-1000:] = part
    hl, hg = (torch.empty(B.sasq_head_bytes(V, H, f), dtype=torch.uint8, device="cuda") for f in (0, 1))
    B.sasq_prepare_head(w, hl, 0)
    B.sasq_prepare_head(w, hg, 1)
    del w
    x = torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16)
    t = torch.tensor([V - 1, V - 1000, V - 7], dtype=torch.int32, device="cuda")
    loss, dx = torch.empty(T, device="cuda"), torch.empty_like(x)
    z = x.double() @ part.double().t()
    at = (t.long() - (V - 1000))[:, None]
    lse = torch.logsumexp(torch.cat((z, torch.full((T, 1), math.log(V - 1000), dtype=torch.float64, device="cuda")), 1), 1, keepdim=True)
    want = (lse - z.gather(1, at))[:, 0]
    p = (z - lse).exp()
    grad = (p.scatter_add(1, at, torch.full_like(at, -1.0, dtype=torch.float64)) @ part.double()) / T
    for piece in (0, 131072):
        B.sasq_linear_ce(x, hl, t, loss, V, B.new_workspace(B.sasq_linear_ce_workspace(T, V, H, True, piece)), dx=dx, head_grad=hg, piece=piece)
        # fp32 sums of 300000 terms, of which 299000 are equal: 2^-24 of the sum a term at most, and 2 H 2^-24 sum |x w| of the logits, 100 for these
        assert ((loss.double() - want).abs() <= 2 * 2 * H * 2.0 ** -24 * 100 + V * 2.0 ** -24).all()
        bound = 2.0 ** -8 * grad.abs() + 2.0 ** -8 * (p @ part.double().abs()) / T * 2 + 0.07 * (grad.abs() + (p @ part.double().abs()) / T)
        assert ((dx.double() - grad).abs() <= bound + 1e-9).all()


def test_other_stream():
    p = Head(128, 3000, 256, "f16", seed=30)
    want = call(p)
    hw = heads(p.w)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = call(p, hw=hw)
    st.synchronize()
    for k in want:
        assert torch.equal(want[k], got[k]), k
