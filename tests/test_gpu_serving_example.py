"""The example that serves an attention block: in steps and all at once the same text gives the same outputs, but for the order of fp32
sums, 16-bit roundings of it, and what the linears' quantizer makes of a rounding that falls on its other side."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_steps_and_all_at_once(int8, dtype):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_attention.py")
    spec = importlib.util.spec_from_file_location("serve_attention", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # q, k, v are the same bits both ways.  An attention output differs by two 16-bit roundings at most (2 u |a|) and so may its code by
    # one; the factor is 2/127 of outputs of size one, so each of 1024 products of o may be off by (2/127 + 2 u) |w|, |w| about 1/32: as
    # independent errors of at most that, 32 * 0.016 / 32 = 0.016 root mean square, five times that for the largest of a million.
    assert example.main(int8=int8, dtype=dtype) < 0.1
