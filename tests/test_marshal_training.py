"""The native marshalling of the calls that keep a byte an element and of the loss, against the checks written out in Python: what it takes gives the same bits
as the call through ctypes, what it does not take raises what the Python checks raise."""
from __future__ import annotations

import pytest
import torch

from paper_2512_14481_amd import binding as B
from tests.test_marshal import broken, outputs

CALLS = list(B._NATIVE_TRAINING)


def arguments(name, dev):
    """Valid arguments of entry point `name` on device `dev` and the positions of its outputs."""
    g = torch.Generator().manual_seed(5)
    M, K, V = 5, 64, 40
    r = lambda *shape, dtype=torch.float16: torch.randn(shape, generator=g).to(dtype).to(dev)
    z = lambda *shape, dtype=torch.float16: torch.zeros(shape, dtype=dtype, device=dev)
    f32, u8, i8 = torch.float32, torch.uint8, torch.int8
    x, y, dy = r(M, K), z(M, K), r(M, K)
    kept = torch.randint(-128, 128, (M, K), generator=g).to(i8).to(dev)
    s, ds, s_k, ds_k = z(1, dtype=f32).add_(0.02), z(1, dtype=f32), z(K, dtype=f32).add_(0.02), z(K, dtype=f32)
    ws = z(1 << 20, dtype=u8)
    if name == "sasq_linear_ce":
        heads = [r(B.sasq_head_bytes(V, K, form) // 2).view(u8) for form in (B.SASQ_HEAD_LOGITS, B.SASQ_HEAD_GRAD)]
        t = torch.tensor([3, -1, 39, 40, 0], dtype=torch.int32).to(dev)
        return (x, heads[0], t, z(M, dtype=f32), V, ws, z(M, dtype=f32), z(1, dtype=f32), y, heads[1], r(M, dtype=f32), 2.0, 0), (3, 6, 7, 8)
    pc = "_pc" in name
    f, df = (s_k, ds_k) if pc else (s, ds)
    one = (kept, dy, y, df) if "bwd" in name else (x, f, y, z(M, K, dtype=i8))
    tail = (ws, 8) if "bwd" in name else (8,)
    return (([one],) + tail, (0,)) if name.endswith("batch") else (one + tail, (2, 3))


@pytest.mark.parametrize("name", CALLS)
def test_host_tensors_and_odd_arguments_are_left_to_the_checks(name):
    B._lib()
    args, _ = arguments(name, "cpu")
    assert getattr(B._native, name)(*args) is None
    assert getattr(B._native, name)() is None and getattr(B._native, name)(*([None] * len(args))) is None
    with pytest.raises(ValueError, match="device tensors"):
        getattr(B, name)(*args)


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_same_bits_and_same_errors_as_through_ctypes(name, monkeypatch):
    B._lib()
    fast = B._native

    def run():
        args, where = arguments(name, "cuda")
        assert getattr(B, name)(*args) is None
        torch.cuda.synchronize()
        return [t.clone() for t in outputs(args, where)]

    assert getattr(fast, name)(*arguments(name, "cuda")[0]) == 0    # taken, not left to the checks
    got = run()
    monkeypatch.setattr(B, "_native", B._Unbound())
    want = run()
    assert len(got) == len(want) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))

    def error(args):
        try:
            getattr(B, name)(*args)
        except Exception as e:                                      # noqa: BLE001 -- compared below
            return type(e), str(e)
        return None

    for args in broken(arguments(name, "cuda")[0]):
        by_ctypes = error(args)
        if by_ctypes is None:
            continue                                                # taken as it is: a length that no check looks at
        with monkeypatch.context() as m:
            m.setattr(B, "_native", fast)
            assert error(args) == by_ctypes
    with monkeypatch.context() as m:                                # the current device is another than the tensors'
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="current device"):
            getattr(B, name)(*arguments(name, "cuda")[0])
