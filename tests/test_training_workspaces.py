"""What the workspaces of a training step's ends are sized for, on the host."""
from __future__ import annotations

import pytest

from paper_2512_14481_amd import binding as B

HEADER = 1024                     # control words of the calls that keep arrival tickets, in front of every workspace


@pytest.mark.parametrize("rows,cols", [(1, 1), (64, 8), (64, 256), (700, 1024)])
def test_control_words_are_not_part_of_what_is_written(rows, cols):
    """Partial sums lie behind the control words, so that a reduction with tickets may follow on the same workspace."""
    chunks = 1 if rows <= 64 else -(-rows // 16)
    assert B.sasq_fakequant_bwd_ckpt_workspace(rows, cols) >= HEADER + 2048 * 8
    assert B.sasq_fakequant_bwd_pc_ckpt_workspace(rows, cols) >= HEADER + 4 * cols * chunks
    for grad in (False, True):
        # left alone: count, ticket, pos, row, tgt, zt, run (2), beta, coef, u, part (2), x (2 bytes, rows of blocks an odd number of 32 columns), each in whole 256 bytes
        up = lambda n: -(-n // 256) * 256
        least = 2 * 256 + 7 * up(4 * rows) + up(8 * rows) + up(-(-rows // 4) * 8) + up(-(-rows // 16) * 16 * (-(-cols // 64) * 2 | 1) * 64)
        assert B.sasq_linear_ce_workspace(rows, 1000, cols, grad) >= HEADER + least


@pytest.mark.parametrize("V,H", [(32000, 4096), (128256, 4096), (100003, 1376), (1000, 256), (513, 2056), (8192, 512), (8200, 64), (1, 1), (4000000, 64), (300000, 8192), (700, 100000)])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("piece", [0, 256, 4096, 1 << 22])
def test_the_longest_batch_is_enough_for_shorter_ones(V, H, grad, piece):
    """A program sizes its workspace once: what a number of rows needs, no smaller number needs more."""
    need, before = B._lib().sasq_linear_ce_workspace, 0
    lengths = [*range(1, 5000), *range(5000, 20000, 37), *range(20000, 140000, 997), *(1 << k for k in range(18, 24))]
    for T in lengths:
        n = need(T, V, H, grad, piece)
        if n == 0:
            assert T * min(piece or 1, V) > 1 << 36 or T * H > 1 << 36        # refused for its size
            continue
        assert n >= before, (T, n, before)
        before = n


def test_what_a_long_batch_needs():
    """No more than the exponentials of a piece, 0.35 GB and 600 bytes a row, with a gradient; the running sums; x once more; M and S."""
    need = B._lib().sasq_linear_ce_workspace
    for T, V, H in ((4096, 32000, 4096), (8192, 32000, 8192), (8192, 128256, 8192), (1 << 17, 32000, 1024), (1 << 20, 32000, 64), (1777, 32000, 5120)):
        Hp = -(-H // 64) * 64
        rest = 2 * T * (Hp + 32) + max(T, 8192 * 1024 // Hp + 256) * Hp * 4 + 64 * T + (1 << 20)
        stats = ((1 << 27) + (5 << 22) + 256 * (T + 63)) / 8                   # 8 bytes for 64 columns and row of a piece: twice 2^26, and a round of tiles more
        assert need(T, V, H, 1, 0) <= 0.35e9 + 600 * T + stats + rest, (T, V, H)
        assert need(T, V, H, 0, 0) <= min(T * V / 8 * 1.01, 1.1e9) + rest


def batch(*shapes):
    arr = (B._CkptItem * len(shapes))()
    for it, (rows, cols) in zip(arr, shapes):
        it.rows, it.cols = rows, cols
    return arr


@pytest.mark.parametrize("pc", ["", "_pc"])
def test_the_largest_batch_of_tensors_is_enough_for_smaller_ones(pc):
    """Fewer tensors, fewer rows, fewer columns: none needs more."""
    need = getattr(B._lib(), f"sasq_fakequant_bwd{pc}_ckpt_batch_workspace")
    for shape in ((64, 256), (700, 1000), (8192, 8192), (1777, 13824)):
        sizes = [need(batch(*[shape] * n), n) for n in range(1, 9)]
        assert sizes[0] > HEADER and sizes == sorted(sizes), (shape, sizes)
    rows = [*range(1, 600), *range(600, 70000, 61), *(1 << k for k in range(17, 25))]
    for cols in (8, 1000, 4096, 40000):
        sizes = [need(batch((r, cols)), 1) for r in rows]
        assert sizes == sorted(sizes), cols
    for r in (64, 1000, 5000):
        sizes = [need(batch((r, c)), 1) for c in range(8, 40000, 56)]
        assert sizes == sorted(sizes), r
