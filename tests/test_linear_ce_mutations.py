"""What the narrow bounds of tests/ce_sharp.py can see, on the host: results of a mistaken kernel, made from the definition in 64 bits, are outside of them at every size.
A row's bounds do not depend on the others, so 260 of a size's rows are enough here."""
from __future__ import annotations

import math

import pytest
import torch

from tests.ce_ref import DT, check
from tests.ce_sharp import PIECES, SIZES, Sharp


def rejected(ref, row, **got):
    """Whether a row of results lies outside."""
    try:
        check(got, {k: (ref[k][0][row], ref[k][1][row]) for k in got})
    except AssertionError:
        return True
    return False


ALL = sorted({(min(s[0], 260), *s[1:3]) for s in SIZES + PIECES}, key=lambda s: s[0] * s[1] * s[2])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H", ALL)
def test_a_mistake_is_outside_the_bounds(T, V, H, dtype):
    p = Sharp(T, V, H, dtype, seed=T + V)
    ref = p.reference()
    check({k: ref[k][0] for k in ref}, ref)
    rows, t, z, zt, others = p.shares()
    w, n = p.w.double(), len(rows)
    q = (z - others[:, None]).exp()
    d = others - zt

    def loss_of(i, lost):                                      # the row's sum without a share `lost` of it
        dd = d[i] + math.log1p(-min(float(lost), 1 - 1e-15))
        return torch.nn.functional.softplus(dd, threshold=1e9)

    mean = q @ w

    def dx_of(i, cols, factor, sums=1.0):                      # some columns' exponentials times `factor`, in the gradient; its S times `sums`
        return torch.sigmoid(d[i]) / n * ((mean[i] + (factor - 1.0) * (q[i, cols] @ w[cols])) / sums - w[t[i]])

    for width in (16, 64, 128):
        groups = -(-V // width)
        share = torch.nn.functional.pad(q, (0, groups * width - V)).view(n, groups, width).sum(2)
        top, row = (share * torch.sigmoid(d)[:, None]).max(0)  # where a group weighs most
        seen = seen_dx = 0
        chosen = range(groups) if groups <= 24 else sorted({*range(0, groups, groups // 16), groups - 1, int(top.argmax())})
        for c in chosen:
            i = int(row[c])
            cols = slice(c * width, min(V, (c + 1) * width))
            lost = loss_of(i, share[i, c])
            seen += rejected(ref, rows[i], loss=lost, lse=zt[i] + lost)
            for factor, sums in ((0.0, 1 - float(share[i, c])), (0.0, 1.0), (2.0, 1.0), (0.25, 1.0)):
                seen_dx += rejected(ref, rows[i], dx=dx_of(i, cols, factor, max(sums, 1e-15)))
        # a group without a column that any row leans on is seen by no bound; where there are rows for all of them, all are seen
        assert seen >= 0.9 * len(chosen) if T >= 16 else seen >= min(len(chosen), 2), (width, seen, len(chosen))
        least = 0.75 if T * 4 >= groups else 0.5 * T / groups
        assert seen_dx >= max(1, least * 4 * len(chosen)), (width, seen_dx, 4 * len(chosen))
    # a part of the contraction that is left out, or added twice; a pass of scaling that misses the first tenth
    def heaviest(cols):                                        # the row that leans on them most
        return int((q[:, cols].sum(1) * torch.sigmoid(d)).argmax())

    for parts in (2, 4, 8):
        for part in range(parts):
            cols = slice(V * part // parts, V * (part + 1) // parts)
            i = heaviest(cols)
            assert all(rejected(ref, rows[i], dx=dx_of(i, cols, factor)) for factor in (0.0, 2.0)), (parts, part)
    cols = slice(0, max(1, V // 10))
    i = heaviest(cols)
    assert rejected(ref, rows[i], dx=dx_of(i, cols, 0.25))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,H", [s for s in ALL if s[0] * s[1] * s[2] < 1 << 33])
def test_what_the_kernels_do_is_inside_the_bounds(T, V, H, dtype):
    """The kernels' steps in torch: fp32 logits and sums, exponentials of 16 bits beside a whole number, dx rounded."""
    p = Sharp(T, V, H, dtype, seed=T + V)
    z = p.z()
    t = p.t.long()[:, None]
    zt = z.gather(1, t)[:, 0].double()
    z.scatter_(1, t, -math.inf)
    top = 11 if dtype == "f16" else 0
    m = (z.amax(1, keepdim=True) * 1.4426950408889634).ceil() - top
    a = torch.exp2(z * 1.4426950408889634 - m)
    s = a.sum(1).double()
    d = (m[:, 0].double() + s.log2()) * math.log(2) - zt
    u = torch.sigmoid(d)
    loss = torch.nn.functional.softplus(d, threshold=1e9)
    dx = (u / T)[:, None] * (a.to(DT[dtype]).float() @ p.w.float() / s[:, None] - p.w.double()[t[:, 0]])
    check({"loss": loss.float(), "lse": (zt + loss).float(), "mean": loss.mean().float().view(1), "dx": dx.to(DT[dtype])}, p.reference())
