"""Cross entropy at the ends of bfloat16's range: heads of large entries whose rows' maxima grow from piece to piece, and targets that are all but certain there.

Tolerances are those of tests/ce_ref.py: a logit that two channels make, the others adding less than 2^-4 of them, is covered by its bound on z.
"""
from __future__ import annotations

import pytest
import torch

from tests.ce_ref import Head, check
from tests.test_gpu_linear_ce import call

pytestmark = pytest.mark.gpu


def large(T, V, H, exponent, rise, seed=0):
    """Channel 0 makes logits that rise by `rise` over the vocabulary; channels from 8 on hold entries around 2^exponent, which x makes small terms of."""
    p = Head(T, V, H, "bf16", seed=seed, sure=0.0)
    p.w, p.x = p.w.float(), p.x.float()
    p.w[:, 0], p.x[:, 0] = torch.linspace(0.0, rise, V), 1.0
    p.w[:, 8:] *= 2.0 ** exponent
    p.x[:, 8:] *= 2.0 ** (-exponent - 10)
    p.w, p.x = p.w.to(torch.bfloat16), p.x.to(torch.bfloat16)
    return p


@pytest.mark.parametrize("T,V,piece", [(40, 1536, 256), (300, 3000, 512), (40, 600, 0), (300, 9000, 0), (2100, 33000, 0)])
@pytest.mark.parametrize("exponent,rise", [(60, 30.0), (75, 120.0), (80, 20.0), (94, 120.0), (94, 5.0), (-80, 30.0)])
def test_large_entries_and_rising_maxima(T, V, piece, exponent, rise):
    """The sums of exponentials times entries stay in fp32 whichever piece a row's largest logit lies in."""
    p = large(T, V, 64, exponent, rise, seed=T)
    ref = p.reference(device="cuda")
    assert torch.isfinite(ref["dx"][0]).all() and ref["dx"][0].abs().max() < 2.0 ** 127
    check(call(p, piece=piece), ref)


@pytest.mark.parametrize("piece", [256, 512, 0])
def test_certain_targets_and_rising_maxima(piece):
    """Losses down to 2^-100 where the other logits rise by 100 from piece to piece: dx keeps its digits."""
    p = large(24, 1536, 64, 0, 100.0, seed=3)
    p.t[:] = 5
    p.w[:, 1] = 0.0
    p.w[5, 1] = 1.0
    p.x[:, 1] = torch.linspace(90.0, 169.0, 24).to(torch.bfloat16)
    ref = p.reference()
    assert ref["loss"][0].min() < 2.0 ** -95 and ref["loss"][0].max() > 1.0
    check(call(p, piece=piece), ref)
