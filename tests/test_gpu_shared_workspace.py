"""One workspace, initialised once, for calls of every kind: the reductions that keep arrival tickets in its control words find them as they left them behind calls
that use the rest of it."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.ce_ref import Head

pytestmark = pytest.mark.gpu
ROWS, COLS = 700, 1024


def reductions(x, dy, s, s_k, ws):
    """What the calls with tickets give, each output NaN before its call."""
    f = lambda n: torch.full((n,), math.nan, device="cuda")
    out = {"absmax": f(1), "ds": f(1), "ds pc": f(COLS), "ds batch 0": f(1), "ds batch 1": f(1)}
    dx = torch.empty_like(dy)
    B.sasq_absmax_scale(x, out["absmax"], ws)
    B.sasq_fakequant_bwd(x, dy, s, dx, out["ds"], ws)
    B.sasq_fakequant_bwd_pc(x, dy, s_k, dx, out["ds pc"], ws)
    B.sasq_fakequant_bwd_batch([(x, dy, s, dx, out["ds batch 0"]), (x, dy, s, None, out["ds batch 1"])], ws)
    torch.cuda.synchronize()
    return out


def keep_a_byte(pc, count):
    need = B.sasq_fakequant_bwd_pc_ckpt_batch_workspace if pc else B.sasq_fakequant_bwd_ckpt_batch_workspace
    bwd = B.sasq_fakequant_bwd_pc_ckpt_batch if pc else B.sasq_fakequant_bwd_ckpt_batch
    items = [(torch.full((ROWS, COLS), 77, dtype=torch.int8, device="cuda"), torch.ones((ROWS, COLS), dtype=torch.float16, device="cuda"), None,
              torch.empty(COLS if pc else 1, device="cuda")) for _ in range(count)]
    return need(items), lambda ws: bwd(items, ws)


def loss(T, V, grad):
    p = Head(T, V, 64, "f16", seed=T)
    heads = []
    for form in (B.SASQ_HEAD_LOGITS, B.SASQ_HEAD_GRAD):
        heads.append(torch.empty(B.sasq_head_bytes(V, 64, form), dtype=torch.uint8, device="cuda"))
        B.sasq_prepare_head(p.w.cuda(), heads[-1], form)
    x, t, out = p.x.cuda(), p.t.cuda(), torch.empty(T, device="cuda")
    mean, dx = torch.empty(1, device="cuda"), torch.empty_like(x) if grad else None
    return B.sasq_linear_ce_workspace(T, V, 64, grad), lambda ws: B.sasq_linear_ce(x, heads[0], t, out, V, ws, mean=mean, dx=dx, head_grad=heads[1] if grad else None)


@pytest.mark.parametrize("kind", ["byte", "byte, three", "byte pc", "byte pc, two", "loss of few rows", "loss of few rows alone", "loss", "loss alone"])
def test_reductions_behind_a_call_without_control_words(kind):
    need, call = {"byte": lambda: keep_a_byte(False, 1), "byte, three": lambda: keep_a_byte(False, 3), "byte pc": lambda: keep_a_byte(True, 1),
                  "byte pc, two": lambda: keep_a_byte(True, 2), "loss of few rows": lambda: loss(20, 700, True), "loss of few rows alone": lambda: loss(20, 700, False),
                  "loss": lambda: loss(300, 9000, True), "loss alone": lambda: loss(300, 9000, False)}[kind]()
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((ROWS, COLS), generator=g, device="cuda").half() for _ in range(2))
    s, s_k = torch.full((1,), 0.02, device="cuda"), torch.full((COLS,), 0.02, device="cuda")
    most = max(B.sasq_absmax_scale_workspace(ROWS, COLS), B.sasq_fakequant_bwd_workspace(ROWS, COLS), B.sasq_fakequant_bwd_pc_workspace(ROWS, COLS),
               B.sasq_fakequant_bwd_batch_workspace(2))
    want = reductions(x, dy, s, s_k, B.new_workspace(most))
    ws = B.new_workspace(max(need, most))
    for _ in range(2):
        got = reductions(x, dy, s, s_k, ws)
        for k in want:
            assert torch.equal(want[k], got[k]), k
        call(ws)
    got = reductions(x, dy, s, s_k, ws)
    for k in want:
        assert torch.equal(want[k], got[k]), k
