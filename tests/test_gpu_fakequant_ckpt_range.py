"""Scale gradients from kept bytes at the ends of bfloat16's range: gradients so large that 252 times a term passes fp32 though the term does not, and so small that
terms lie near its smallest step.

Tolerance: that of tests/test_gpu_fakequant_ckpt.py, and for each term 2^-139, what a product below fp32's normal numbers may lose.
"""
from __future__ import annotations

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.test_gpu_fakequant_ckpt import calls, ds_of

pytestmark = pytest.mark.gpu


def inputs(rows, cols, size):
    g = torch.Generator().manual_seed(rows + cols)
    kept = torch.randint(-126, 127, (rows, cols), generator=g).to(torch.int8)
    dy = torch.randn((rows, cols), generator=g) * 2.0 ** (size - 14)
    some = torch.randperm(rows * cols, generator=g)[:max(1, rows * cols // 500)]
    k, d, n = kept.view(-1), dy.view(-1), torch.arange(len(some))
    k[some] = torch.where(n % 2 == 0, 127, -128).to(torch.int8)                 # clamped, and of the largest gradients
    d[some] = torch.where(n % 4 < 2, 1.0, -1.0) * 1.5 * 2.0 ** size
    k[:2], d[:2] = torch.tensor([126, -100], dtype=torch.int8)[:len(k)], torch.tensor([1.0, 1.0])[:len(k)] * 2.0 ** (size + 8)
    return kept, dy.to(torch.bfloat16)


def check(ds, kept, dy, bits, pc):
    want, tol = ds_of(kept, dy, bits, pc)
    assert want.abs().max() < 2.0 ** 127
    off = (ds.cpu().double() - want).abs()
    assert (off <= tol + 2.0 ** -139 * (kept.shape[0] if pc else kept.numel())).all(), (off.max(), tol[off.argmax()])


SIZES = [(1, 1), (3, 8), (64, 256), (129, 33), (700, 1000), (777, 1001), (2100, 512)]


@pytest.mark.parametrize("size", [114, 0, -100, -117])
@pytest.mark.parametrize("bits", [8, 2])
@pytest.mark.parametrize("pc", [False, True])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_large_and_small_gradients(rows, cols, pc, bits, size):
    kept, dy = inputs(rows, cols, size)
    _, bwd, need = calls(pc)
    k, d = kept.cuda(), dy.cuda()
    dx, ds = torch.empty_like(d), torch.full((cols if pc else 1,), torch.nan, device="cuda")
    bwd(k, d, dx, ds, B.new_workspace(need(rows, cols)), bits)
    check(ds, kept, dy, bits, pc)
    assert torch.equal(dx.cpu().view(torch.int16), torch.where(kept.short().abs() <= 126, dy, 0).view(torch.int16))


@pytest.mark.parametrize("pc", [False, True])
def test_large_gradients_in_a_batch(pc):
    t = [inputs(r, c, 114) for r, c in ((64, 256), (700, 1000), (2100, 512))]
    items = [(k.cuda(), d.cuda(), None, torch.full((k.shape[1] if pc else 1,), torch.nan, device="cuda")) for k, d in t]
    ws = B.new_workspace((B.sasq_fakequant_bwd_pc_ckpt_batch_workspace if pc else B.sasq_fakequant_bwd_ckpt_batch_workspace)(items))
    (B.sasq_fakequant_bwd_pc_ckpt_batch if pc else B.sasq_fakequant_bwd_ckpt_batch)(items, ws)
    for (kept, dy), it in zip(t, items):
        check(it[3], kept, dy, 8, pc)
