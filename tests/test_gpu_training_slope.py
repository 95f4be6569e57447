"""The factors' gradients of a whole training step against differences of the loss, with bounds that are small beside the gradients themselves.

What the straight-through estimator holds fixed is held at what the kernels had: each layer's input h, its quantized input y, its mask m and kept bytes v (c / 252
inside the range, the ends outside).  A step's loss then is, in 64 bits, a function of the factors f around s,
    y' = y + m (h' - h) + (f - s) v        h'' = h2 + (y' - y) W^T        loss(h'')
whose slope at s is the gradient; nothing of the forward's roundings is left.  The backward's are, each at most half a step of its tensor:
    dh      what tests/ce_ref.py allows            dy of a layer: its products in fp32, 2 n 2^-24 of the sum of their sizes, and a rounding to 16 bits
and of the slope each takes its sum with the sizes of what it is multiplied with on the way to ds.
"""
from __future__ import annotations

import math

import pytest
import torch

from tests.ce_ref import HALF, Head
from tests.test_gpu_training_step import example

pytestmark = pytest.mark.gpu
LIMIT = 2.0 ** -25


def slopes_and_bounds(net, dtype, directions):
    """For each layer and direction of its factors: the slope by differences, its bound, and what the kernels say."""
    D = lambda t: t.cpu().double()
    w, s, y, h = [D(la.w) for la in net.layers], [D(la.s) for la in net.layers], [D(la.xq) for la in net.layers], [D(net.x)]
    h.append(D((net.layers[0].xq @ net.layers[0].w.t())))
    end = D(net.h)
    assert torch.equal(end, D(net.layers[1].xq @ net.layers[1].w.t()))
    kept = [la.kept.cpu() for la in net.layers]
    m = [((k != 127) & (k != -128)).double() for k in kept]
    v = [torch.where(k == 127, 127.0, torch.where(k == -128, -128.0, k.double() / 252)) for k in kept]
    rows = net.targets.cpu() >= 0
    t, head = net.targets.cpu().long()[rows], D(net.w)

    def loss(moved):
        y0 = moved[0] * v[0]                                                # y' - y
        y1 = m[1] * (y0 @ w[0].t()) + moved[1] * v[1]
        z = (end + y1 @ w[1].t())[rows] @ head.t()
        return (torch.logsumexp(z, 1) - z[torch.arange(len(t)), t]).mean()

    p = Head(*net.x.shape[:1], net.vocab, net.x.shape[1], dtype)
    p.x, p.w, p.t = net.h.cpu(), net.w.cpu(), net.targets.cpu()
    dh, e_dh = p.reference(scale=net.scale)["dx"]
    eps, out = HALF[dtype], []
    product = lambda a, b: (a @ b, 2 * a.shape[1] * 2.0 ** -24 * (a.abs() @ b.abs()))
    dy1, r1 = product(dh, w[1])
    r1 = r1 + eps * dy1.abs() * 1.02 + LIMIT
    dy0, r0 = product(m[1] * dy1, w[0])
    r0 = r0 + eps * dy0.abs() * 1.02 + LIMIT
    for i, layer in enumerate(net.layers):
        for direction in directions(layer.s.numel()):
            u = v[i] * direction
            # what each element of dy of this layer, of the layer behind it, and of dh is multiplied with
            if i == 1:
                bound = (r1 * u.abs()).sum() + (e_dh * (u @ w[1].t()).abs()).sum()
            else:
                back = m[1] * (u @ w[0].t())
                bound = (r0 * u.abs()).sum() + (r1 * back.abs()).sum() + (e_dh * (back @ w[1].t()).abs()).sum()
            moved = [torch.zeros(1, dtype=torch.float64)] * 2
            ends = []
            step = 1e-4 * s[i].abs().mean() * direction
            for k in (1.0, 0.5):
                moved[i] = k * step
                up = loss(moved)
                moved[i] = -k * step
                ends.append((up - loss(moved)) / (2 * k * 1e-4 * s[i].abs().mean()))
            got = (D(layer.ds) * direction).sum() / net.scale
            # fp32 sums of ds: 8 2^-24 of the terms, as in tests/test_gpu_fakequant_ckpt.py; truncation of the differences: four thirds of what halving changes
            dy = (dy0, dy1)[i]
            bound = (bound + 10 * 2.0 ** -24 * (dy * u).abs().sum()) / net.scale + 1.4 * abs(ends[0] - ends[1]) + 1e-10
            out.append((ends[1].item(), bound.item(), got.item()))
    return out


@pytest.mark.parametrize("per_channel", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_slopes(dtype, per_channel):
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    found = []
    for seed in range(6):
        net = example().Network(60, 64, 96, 300, dt, per_channel, seed=seed)
        for layer in net.layers:
            layer.s *= 0.6                                                  # some clamping
        net.step()
        torch.cuda.synchronize()
        g = torch.Generator().manual_seed(seed)
        some = lambda n: [torch.ones(1, dtype=torch.float64)] if n == 1 else [torch.randn(n, generator=g).double().sign() for _ in range(4)] + [
            torch.eye(n, dtype=torch.float64)[k] for k in (0, n // 2, n - 1)]
        found += slopes_and_bounds(net, dtype, some)
    size = lambda values: math.sqrt(sum(a * a for a in values))
    # gradients that are nought, or another sign, would be outside
    assert size([b for _, b, _ in found]) < size([a for a, _, _ in found]) / 4
    for slope, bound, got in found:
        assert abs(got - slope) <= bound, (slope, bound, got)
