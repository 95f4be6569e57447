"""A scale-training step made of the calls that belong to it: fake-quant with a byte kept, frozen linears, the loss at the head, the way back; and the example that
runs it.  Each stage is held against its definition in 64 bits, computed from what the stage before it gave."""
from __future__ import annotations

import importlib.util
import math
import os

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.ce_ref import HALF, Head, check
from tests.test_gpu_fakequant_ckpt import bytes_of, check_ds

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_scales.py")
    spec = importlib.util.spec_from_file_location("train_scales", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("per_channel", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_stages(dtype, per_channel):
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    net = example().Network(100, 128, 352, 700, dt, per_channel, seed=3)
    net.step()
    torch.cuda.synchronize()
    x = net.x.cpu()
    for layer in net.layers:
        kept, q = bytes_of(x, layer.s.cpu(), 8)
        assert torch.equal(layer.kept.cpu(), kept)
        assert torch.equal(layer.xq.cpu(), (q.float() * layer.s.cpu()).to(dt))
        x = (layer.xq @ layer.w.t()).cpu()
    assert torch.equal(x, net.h.cpu())
    p = Head(100, 700, 128, dtype)
    p.x, p.w, p.t = x, net.w.cpu(), net.targets.cpu()
    check({"loss": net.loss, "mean": net.mean, "dx": net.dh}, p.reference(scale=net.scale))
    d = net.dh.cpu()
    for layer in reversed(net.layers):
        exact = d.double() @ layer.w.cpu().double()
        n = d.shape[1]
        dy = torch.empty_like(layer.dx)
        B.sasq_linear_bwd_input(d.cuda(), layer.wt, dy, dy.shape[1])
        tol = n * 2.0 ** -24 * (d.double().abs() @ layer.w.cpu().double().abs()) + HALF[dtype] * exact.abs() * 1.01 + 2.0 ** -25
        assert ((dy.cpu().double() - exact).abs() <= tol).all()
        kept = layer.kept.cpu()
        keep = (kept != 127) & (kept != -128)
        assert torch.equal(layer.dx.cpu(), torch.where(keep, dy.cpu(), 0))
        check_ds(layer.ds, kept, dy.cpu(), 8, per_channel)
        d = layer.dx.cpu()


@pytest.mark.parametrize("per_channel", [False, True])
def test_captured_steps(per_channel):
    """Replays with factors that move between them give what eager steps give, bit for bit."""
    module = example()
    a, b = (module.Network(100, 128, 352, 700, torch.bfloat16, per_channel, seed=1) for _ in range(2))
    b.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    for i in range(4):
        a.step()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.loss, b.loss) and torch.equal(a.mean, b.mean) and torch.equal(a.dh, b.dh)
        for la, lb in zip(a.layers, b.layers):
            assert torch.equal(la.ds, lb.ds) and torch.equal(la.dx, lb.dx)
        for net in (a, b):
            net.update(i + 1, 1e-3)


def test_slope_along_the_factors():
    """The factors' gradients against differences of the loss, with what the straight-through estimator holds fixed held fixed: x' = x + s e inside the range,
    s q outside, e and q as at the start, all in 64 bits."""
    net = example().Network(60, 64, 96, 300, torch.bfloat16, False, seed=5)
    for layer in net.layers:
        layer.s *= 0.6                                                  # some clamping
    net.step()
    torch.cuda.synchronize()
    w = [layer.w.cpu().double() for layer in net.layers]
    held, x = [], net.x.cpu().double()
    for layer, wi in zip(net.layers, w):
        s = layer.s.cpu().double()
        r = x / s
        q = r.round().clamp(-128, 127)
        held.append((r.round() == q, q - r, q))
        x = torch.where(held[-1][0], x + s * held[-1][1], s * q) @ wi.t()
    rows = net.targets.cpu() >= 0
    t = net.targets.cpu().long()[rows]

    def loss(factors):
        h = net.x.cpu().double()
        for (inside, e, q), wi, s in zip(held, w, factors):
            h = torch.where(inside, h + s * e, s * q) @ wi.t()
        z = h[rows] @ net.w.cpu().double().t()
        return (torch.logsumexp(z, 1) - z[torch.arange(len(t)), t]).mean()

    base = [layer.s.cpu().double() for layer in net.layers]
    for i, layer in enumerate(net.layers):
        step = base[i] * 1e-4
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + step, base[i] - step
        slope = ((loss(up) - loss(down)) / (2 * step)).item()
        # what the 16-bit roundings of activations and gradients, and the bytes', add are independent terms of the size of the sum's: per element of dy, 2^-8 of
        # rounding in each of four tensors and 1/504 of the byte, against terms of |dy| * 0.29; the sum of n such errors has the root of n of them
        dy = torch.empty_like(layer.dx)
        d = net.dh if i == 1 else net.layers[1].dx
        B.sasq_linear_bwd_input(d, layer.wt, dy, dy.shape[1])
        noise = dy.cpu().double().norm().item() * (4 * 2.0 ** -8 + 1 / 504) * 128
        assert math.isfinite(slope) and abs(layer.ds.item() / net.scale - slope) < noise, (layer.ds.item(), slope, noise)


@pytest.mark.parametrize("per_channel", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_example_runs(dtype, per_channel):
    assert all(math.isfinite(v) for v in example().main(steps=3, per_channel=per_channel, dtype=dtype))
