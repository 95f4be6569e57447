"""Cases of the cross entropy whose bounds stay narrow where rows are long: logits that are exact in fp32, and rows that lean on few columns of the vocabulary.

x holds whole numbers of size 2 at most, W whole numbers of size 3 at most times a power of two that brings the logits to a standard deviation of about 4.  Products
and their sums, in any order, are whole numbers under 2^24 times that power (6 H < 2^24): z has no error at all.  What is left, per element, with u32 = 2^-24:
  a_v   exponent z log2(e) - M: its product is rounded once, log2(e) is off by 2^-26 of itself, 2^x by one unit in the last place:
        ea = ln 2 (2^-24 (2 Z + 12) + 2^-26 Z) + 2^-23, Z the largest |z| log2(e) of the row (M is at most 12 past it)
  S     fp32 sums of positive numbers, a number in DEPTH of them at most: 34 of a tile's lane and its neighbours, 16 groups a thread, 22 of threads and waves, one
        a piece; 128 in all
  d     ed = ea + (DEPTH + 2) u32;  loss off by u ed, lse by ed, and both by a rounding
  dx    the 16-bit exponentials are off by eps relative, in fp16 also by 2^-35 of the row's sum each, twice where they are scaled; fp32 sums over V, doubled
        for the matrix unit's own roundings; u and S by ed; one rounding to 16 bits
A row's largest columns hold tenths of its sum, so a group of columns, a part of the contraction or a factor that is lost is far outside.
"""
from __future__ import annotations

import math

import torch

from tests.ce_ref import DT, HALF, TINY

U32, DEPTH = 2.0 ** -24, 128


class Sharp:
    def __init__(self, T, V, H, dtype="f16", seed=0, left_out=0.0, device="cpu"):
        assert 6 * H < 1 << 24
        g = torch.Generator().manual_seed(seed)
        self.T, self.V, self.H, self.dtype, self.device = T, V, H, dtype, device
        power = round(math.log2(math.sqrt(8 * H) / 4))                             # var x = 2, var of W's whole numbers 4
        self.w = (torch.randint(-3, 4, (V, H), generator=g).float() * 2.0 ** -power).to(DT[dtype])
        self.x = torch.randint(-2, 3, (T, H), generator=g).float().to(DT[dtype])
        t = torch.randint(V, (T,), generator=g)
        z = self.z()
        sure = torch.arange(T) % 3 == 0                                            # their target is the largest column of all
        t = torch.where(sure, z.argmax(1).cpu(), t)
        out = torch.rand(T, generator=g) < left_out
        self.t = torch.where(out, torch.where(torch.arange(T) % 2 == 0, -100, V + 3), t).to(torch.int32)

    def z(self):
        return self.x.to(self.device).float() @ self.w.to(self.device).float().t()         # exact

    def shares(self, zeros=0):
        """For the counted rows: their numbers, targets, logits of the others and of the target (64 bits), and the others' logarithmic sum, with so many logits of 0 more."""
        t = self.t.to(self.device)
        rows = ((t >= 0) & (t < self.V)).nonzero()[:, 0]
        t = t[rows].long()
        z = self.z()[rows].double()
        zt = z.gather(1, t[:, None])[:, 0]
        z.scatter_(1, t[:, None], -math.inf)
        others = torch.logsumexp(z, 1)
        if zeros:
            others = torch.logaddexp(others, torch.full_like(others, math.log(zeros)))
        return rows, t, z, zt, others

    def reference(self, scale=1.0, zeros=0):
        """{name: (values, tolerance)}, in 64 bits; of a head with so many entries of nothing but zeros in front."""
        rows, t, z, zt, others = self.shares(zeros)
        T, H, V = self.T, self.H, self.V
        zero = lambda *s: torch.zeros(s, dtype=torch.float64, device=self.device)
        loss, lse, dx, e_loss, e_lse, e_dx = zero(T), zero(T), zero(T, H), zero(T), zero(T), zero(T, H)
        if len(rows):
            w = self.w.to(self.device).double()
            d = others - zt
            u = torch.sigmoid(d)
            loss[rows] = torch.nn.functional.softplus(d, threshold=1e9)
            lse[rows] = zt + loss[rows]
            most = torch.maximum(z.masked_fill(z == -math.inf, 0).abs().amax(1), zt.abs()) * 1.4427
            ea = 0.6932 * (U32 * (2 * most + 12) + U32 / 4 * most) + 2 * U32
            ed = ea + (DEPTH + 2) * U32
            e_loss[rows] = u * ed * 1.01 + U32 * loss[rows] + 1e-30
            e_lse[rows] = ed + U32 * lse[rows].abs()
            q = (z - others[:, None]).exp().nan_to_num(0.0)
            g = scale / len(rows)
            mean_w, mean_abs, eps = q @ w, q @ w.abs(), HALF[self.dtype]
            dx[rows] = g * u[:, None] * (mean_w - w[t])
            flush = V * 2.0 ** -34 * w.abs().max() if self.dtype == "f16" else 0.0
            e_dx[rows] = abs(g) * u[:, None] * ((eps + 2 * ea + 2 * V * U32)[:, None] * mean_abs + flush + (2 * ed[:, None] + 8 * U32) * (mean_w - w[t]).abs()) * 1.01
            e_dx[rows] += eps * dx[rows].abs() * 1.01 + TINY[self.dtype]
        n = max(len(rows), 1)
        mean = loss.sum() / n
        return {"loss": (loss, e_loss), "lse": (lse, e_lse), "mean": (mean.view(1), (e_loss.sum() / n + U32 * mean).view(1)), "dx": (dx, e_dx)}


# one of each kind of call: tiles, large and small, whole rounds and halves, in one piece and several, contractions in parts, few rows with 16, 32 and 64 columns a workgroup,
# many rows of small heads; long and short rows
SIZES = [(520, 9000, 4096), (1100, 16001, 4096), (2100, 9000, 2048), (129, 33000, 1024), (3000, 24000, 320), (384, 30000, 1024), (640, 9000, 2048), (257, 33000, 520),
         (300, 8193, 333), (100, 9000, 256), (1, 300, 4097), (3, 8300, 4096), (16, 8192, 2049), (17, 300, 2048), (33, 2049, 2113), (64, 8200, 2048), (64, 1000, 256),
         (193, 1000, 2048), (500, 513, 2056), (1000, 700, 256), (4200, 8500, 512)]
PIECES = [(600, 9000, 2048, 2304), (300, 2817, 192, 512), (50, 4100, 4096, 1024)]
