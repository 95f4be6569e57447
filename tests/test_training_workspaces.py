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
