"""The cross entropy of a frozen head in 64 bits on the host, and how far the kernels may be from it.

Tolerances, per element, with eps half a step of the 16-bit type and n the length of a sum (fp32 sums in any order are off by at most n 2^-24 of the sum of the
terms' sizes; doubled for the matrix unit's own intermediate roundings):
  z     2 H 2^-24 sum_h |x W|  =: ez (the largest of the row)
  lse   2 ez (numerator and target) and the sum over V, its logarithm and the rounding of the result: (V + 8) 2^-24 + 2^-24 |lse|
  loss  d = lse_o - z_t is off by that; loss = ln(1 + e^d) by at most u times as much, and 2^-24 of itself
  dx    the average of W over the others is off by eps (exponentials in 16 bits, relative) + 2 (2 ez + 2^-20) + 2 V 2^-24 of sum q |W|, in fp16 also by
        V 2^-34 max |W| (two roundings to the smallest step, 2^-24, beside a largest exponential of 2^10 at least);
        u by what d is off by; then one rounding, and the type's smallest step
"""
from __future__ import annotations

import math

import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}


class Head:
    def __init__(self, T, V, H, dtype="f16", seed=0, left_out=0.0, sure=9.0, scale=1.3):
        g = torch.Generator().manual_seed(seed)
        self.T, self.V, self.H, self.dtype = T, V, H, dtype
        self.w = (torch.randn((V, H), generator=g) * scale / math.sqrt(H)).to(DT[dtype])
        t = torch.randint(V, (T,), generator=g)
        x = torch.randn((T, H), generator=g) + torch.rand((T, 1), generator=g) * sure * self.w[t].float()
        self.x = x.to(DT[dtype])
        out = torch.rand(T, generator=g) < left_out
        self.t = torch.where(out, torch.where(torch.arange(T) % 2 == 0, -100, V + 3), t).to(torch.int32)

    def reference(self, row_weight=None, scale=1.0, device="cpu"):
        """{name: (values, tolerance)}, in 64 bits."""
        x, w, T, V, H = self.x.to(device).double(), self.w.to(device).double(), self.T, self.V, self.H
        rows = ((self.t.to(device) >= 0) & (self.t.to(device) < V)).nonzero()[:, 0]
        zero = lambda *s: torch.zeros(s, dtype=torch.float64, device=device)
        loss, lse, dx, e_loss, e_lse, e_dx = zero(T), zero(T), zero(T, H), zero(T), zero(T), zero(T, H)
        if len(rows):
            t, xr, i = self.t.to(device)[rows].long(), x[rows], torch.arange(len(rows), device=device)
            z, u32 = xr @ w.t(), 2.0 ** -24
            ez = 2 * H * u32 * (xr.abs() @ w.abs().t()).amax(1)
            zt = z[i, t]
            z[i, t] = -math.inf
            others = torch.logsumexp(z, 1)
            d = others - zt
            u = torch.sigmoid(d)
            loss[rows] = torch.nn.functional.softplus(d, threshold=1e9)
            lse[rows] = zt + loss[rows]
            ed = 2 * ez + (V + 8) * u32 + u32 * others.abs().clamp(min=0, max=1e30)
            e_loss[rows] = u * ed * 1.01 + u32 * loss[rows] + 1e-30
            e_lse[rows] = ed + u32 * lse[rows].abs()
            q = torch.softmax(z, 1).nan_to_num(0.0)
            g = scale * (torch.full((T,), 1.0 / len(rows), dtype=torch.float64, device=device) if row_weight is None else row_weight.to(device).double())[rows, None]
            eps = HALF[self.dtype]
            dx[rows] = g * u[:, None] * (q @ w - w[t])
            rel = (eps + 2 * (2 * ez + 2.0 ** -20) + 2 * V * u32)[:, None]
            flush = V * 2.0 ** -34 * w.abs().max() if self.dtype == "f16" else 0.0
            e_dx[rows] = (g * u[:, None]).abs() * (rel * (q @ w.abs()) + flush + (2 * ed[:, None] + 8 * u32) * (q @ w - w[t]).abs()) * 1.01
            e_dx[rows] += eps * dx[rows].abs() * 1.01 + TINY[self.dtype]
        n = max(len(rows), 1)
        mean = loss.sum() / n
        return {"loss": (loss, e_loss), "lse": (lse, e_lse), "mean": (mean.view(1), (e_loss.sum() / n + 2.0 ** -24 * mean).view(1)), "dx": (dx, e_dx)}


def check(got, ref, names=None):
    for name, value in got.items():
        if value is None:
            continue
        want, tol = ref[name]
        v = value.detach().to(want.device).double().view(want.shape)
        off = (v - want).abs()
        bad = ~(off <= tol)
        assert not bad.any(), (name, int(bad.sum()), "of", bad.numel(), "first", bad.nonzero()[0].tolist(), v[bad][:3].tolist(), want[bad][:3].tolist(),
                               tol[bad][:3].tolist())
