"""The tile of the cross entropy's gradient product, a host function of the library: each where it was measured the faster one."""
from __future__ import annotations

import ctypes

import pytest

from tests.dispatch import _function


def grad_tile(rows, channels, columns):
    """Rows and columns of the gradient's tile, for so many columns of a piece (sasq::ce_grad_tile)."""
    i64 = ctypes.c_int64
    return (256, 128, 128)[_function("_ZN4sasq12ce_grad_tileElll", i64, i64, i64)(rows, channels, columns)]


@pytest.mark.parametrize("columns", [1024, 2048, 4096, 6144, 8192])
def test_a_half_of_a_short_contraction_costs_a_whole_tile(columns):
    """300 x 4096 -> 1000 takes 55 us by 128x128 and 70 by 256x256 with halves."""
    assert grad_tile(300, 4096, columns) == grad_tile(384, 4096, columns) == 128


def test_halves_of_long_contractions():
    assert grad_tile(350, 2048, 100096) == grad_tile(384, 4096, 20224) == grad_tile(4200, 4096, 20480) == 256
    assert grad_tile(333, 1376, 100096) == grad_tile(300, 1000, 60160) == 128


def test_whole_tiles():
    for columns in (1024, 8192, 32000):
        assert grad_tile(256, 4096, columns) == grad_tile(4096, 4096, columns) == 256
