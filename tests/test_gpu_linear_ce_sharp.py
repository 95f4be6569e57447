"""Cross entropy of long rows with logits that are exact, within bounds narrow enough to see a lost group of columns, part or factor (tests/test_linear_ce_mutations.py)."""
from __future__ import annotations

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.ce_ref import DT, check
from tests.ce_sharp import PIECES, SIZES, Sharp
from tests.test_gpu_linear_ce import call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H", SIZES)
def test_exact_logits(T, V, H, dtype, grad):
    p = Sharp(T, V, H, dtype, seed=T + V, device="cuda")
    check(call(p, grad=grad, scale=64.0), p.reference(scale=64.0))


@pytest.mark.parametrize("left_out", [0.1, 0.6])
@pytest.mark.parametrize("T,V,H", [s for s in SIZES if s[0] > 60])
def test_exact_logits_with_rows_left_out(T, V, H, left_out):
    p = Sharp(T, V, H, "bf16", seed=T, left_out=left_out, device="cuda")
    check(call(p, scale=64.0), p.reference(scale=64.0))


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H,piece", PIECES)
def test_exact_logits_in_pieces(T, V, H, piece, dtype, grad):
    p = Sharp(T, V, H, dtype, seed=T, left_out=0.1, device="cuda")
    check(call(p, piece=piece, grad=grad, scale=64.0), p.reference(scale=64.0))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_exact_logits_at_far_offsets(dtype):
    """The last thousand entries of a vocabulary of 300000 by 4096 channels, 2.4 GB a layout, behind zeros: those add their number to the sums, and nothing to any
    other (their products are zeros, so that the contraction rounds as often as that of a thousand)."""
    T, V, H = 5, 300000, 4096
    far = Sharp(T, 1000, H, dtype, seed=9, device="cuda")
    w = torch.zeros((V, H), dtype=DT[dtype], device="cuda")
    w[-1000:] = far.w.cuda()
    hl, hg = (torch.empty(B.sasq_head_bytes(V, H, f), dtype=torch.uint8, device="cuda") for f in (0, 1))
    B.sasq_prepare_head(w, hl, 0)
    B.sasq_prepare_head(w, hg, 1)
    del w
    ref = far.reference(zeros=V - 1000)
    x, t = far.x.cuda(), far.t.cuda() + (V - 1000)
    for piece in (0, 131072):
        out = {"loss": torch.empty(T, device="cuda"), "lse": torch.empty(T, device="cuda"), "mean": torch.empty(1, device="cuda"), "dx": torch.empty_like(x)}
        B.sasq_linear_ce(x, hl, t, out["loss"], V, B.new_workspace(B.sasq_linear_ce_workspace(T, V, H, True, piece)), lse=out["lse"], mean=out["mean"], dx=out["dx"],
                         head_grad=hg, piece=piece)
        check(out, ref)
