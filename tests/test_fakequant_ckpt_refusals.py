"""What the fake-quant calls that keep a byte refuse, on the host before anything is launched, and their workspaces."""
from __future__ import annotations

import pytest
import torch

from paper_2512_14481_amd import binding as B

P = 0x10000                       # never read: every call below is refused first
NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
GOOD = dict(x=P, s=P, out=P, kept=P, dy=P, ds=P, rows=8, cols=64)


def items(*changes):
    arr = (B._CkptItem * max(len(changes), 1))()
    for i, c in enumerate(changes):
        for k, v in dict(GOOD, **c).items():
            setattr(arr[i], k, v)
    return arr


@pytest.mark.parametrize("pc", ["", "_pc"])
def test_items(pc):
    lib = B._lib()
    fwd = lambda *c, n=None, bits=8, dt=0: getattr(lib, f"sasq_fakequant_fwd{pc}_ckpt_batch")(items(*c), len(c) if n is None else n, bits, dt, None)
    bwd = lambda *c, n=None, bits=8, dt=0, ws=P, wsb=1 << 40: getattr(lib, f"sasq_fakequant_bwd{pc}_ckpt_batch")(
        items(*c), len(c) if n is None else n, bits, dt, ws, wsb, None)
    both = [(dict(kept=None), NULL), (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=1 << 40, cols=2), SHAPE), (dict(kept=P + 8), ALIGN),
            (dict(out=P + 2), ALIGN)]
    for change, rc in both + [(dict(x=None), NULL), (dict(s=None), NULL), (dict(out=None), NULL), (dict(x=P + 2), ALIGN)]:
        assert fwd(change) == rc and fwd({}, change) == rc, change
    for change, rc in both + [(dict(dy=None), NULL), (dict(ds=None), NULL), (dict(dy=P + 2), ALIGN)]:
        assert bwd(change) == rc and bwd({}, change) == rc, change
    for call in (fwd, bwd):
        assert call({}, n=0) == call({}, n=9) == SHAPE
        assert call({}, bits=1) == call({}, bits=9) == call({}, dt=2) == UNSUPPORTED
    if pc:
        assert fwd(dict(cols=(1 << 24) + 1)) == SHAPE
        assert fwd(*[dict(rows=1 << 13, cols=1 << 24)] * 8) == SHAPE
    need = getattr(lib, f"sasq_fakequant_bwd{pc}_ckpt_batch_workspace")
    n = need(items({}, dict(rows=5000)), 2)
    assert n > 0 and bwd({}, dict(rows=5000), wsb=n - 1) == WORKSPACE and bwd({}, ws=None) == WORKSPACE and bwd({}, ws=P + 8) == ALIGN
    assert need(items({}), 0) == need(items({}), 9) == need(items(dict(rows=0)), 1) == need(None, 1) == 0
    assert getattr(lib, f"sasq_fakequant_fwd{pc}_ckpt_batch")(None, 1, 8, 0, None) == NULL


@pytest.mark.parametrize("pc", ["", "_pc"])
def test_single_calls(pc):
    lib = B._lib()
    fwd, bwd = getattr(lib, f"sasq_fakequant_fwd{pc}_ckpt"), getattr(lib, f"sasq_fakequant_bwd{pc}_ckpt")
    assert fwd(None, P, P, P, 8, 8, 8, 0, None) == fwd(P, None, P, P, 8, 8, 8, 0, None) == fwd(P, P, None, P, 8, 8, 8, 0, None) == fwd(P, P, P, None, 8, 8, 8, 0, None) == NULL
    assert bwd(None, P, P, P, 8, 8, 8, 0, P, 1 << 30, None) == bwd(P, None, P, P, 8, 8, 8, 0, P, 1 << 30, None) == bwd(P, P, P, None, 8, 8, 8, 0, P, 1 << 30, None) == NULL
    need = getattr(B, f"sasq_fakequant_bwd{pc}_ckpt_workspace")
    assert bwd(P, P, P, P, 800, 64, 8, 0, P, need(800, 64) - 1, None) == WORKSPACE
    assert need(0, 8) == need(8, 0) == 0 and need(1 << 20, 4096) > 0


def test_binding():
    x, k, s = torch.zeros((4, 8), dtype=torch.float16), torch.zeros((4, 8), dtype=torch.int8), torch.zeros(1)
    with pytest.raises(ValueError):
        B.sasq_fakequant_fwd_ckpt(x, s, x, k)                          # host tensors
    with pytest.raises(ValueError):
        B.sasq_fakequant_fwd_ckpt(x, s, x, k[:3])
    with pytest.raises(TypeError):
        B.sasq_fakequant_fwd_ckpt(x, s, x, x)
    with pytest.raises(ValueError):
        B.sasq_fakequant_fwd_pc_ckpt(x, s, x, k)
    with pytest.raises(ValueError):
        B.sasq_fakequant_fwd_ckpt_batch([])
    with pytest.raises(ValueError):
        B.sasq_fakequant_bwd_ckpt_batch([(k, x, x[:3], s)], k)
