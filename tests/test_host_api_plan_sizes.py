"""The entry points over a plan go by the plan's sizes, not by the shapes that the tensors happen to have (CPU)."""
import ctypes

import pytest
import torch

from paper_2609_35110_b200 import binding as B
from paper_2609_35110_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build_mod.build_library()
    return B._lib()


class OnDevice:
    """A CPU tensor that says it is on the device: everything up to the C call can be exercised without one."""

    def __init__(self, t):
        self.t = t
        self.is_cuda, self.dtype, self.shape, self.device = True, t.dtype, t.shape, t.device

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def calls(monkeypatch):
    """Records the forward calls instead of making them."""
    made = []

    class Lib:
        def __getattr__(self, name):
            if not name.startswith("sol_attn3d_forward"):
                return getattr(built, name)

            def call(*args):
                made.append(name)
                return 0
            return call

    built = B._lib()
    monkeypatch.setattr(B, "_lib", lambda: Lib())
    monkeypatch.setattr(B, "_check_on_device", lambda *t: None)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    return made


def tensors(*shape, dtype=torch.bfloat16):
    return OnDevice(torch.zeros(*shape, dtype=dtype))


def test_plan_dims():
    p = B.sol_attn3d_plan_ex([(3, 2, 4, 5), (7, 0, 1, 1)], 6, 64, (16, 24, 24))
    assert B.sol_attn3d_plan_dims(p) == (2, 6, 64, 50)
    assert B._lib().sol_attn3d_plan_dims(None, (ctypes.c_int64 * 4)()) == B.ERR_INVALID_ARG
    assert B._lib().sol_attn3d_plan_dims(p, None) == B.ERR_INVALID_ARG
    B.sol_attn3d_destroy(p)


def test_linear_decays_and_states_are_the_plans(calls):
    """q seen as [tokens, 2 heads of 128] under a plan of 4 heads of 64: two decays would be read as four."""
    p = B.sol_attn3d_plan_ex([(10, 0, 1, 1)], 4, 64, (16, 24, 24))
    f32 = torch.float32

    def call(q=(10, 4, 64), decay=4, state=None, tokens=10):
        x = tensors(*q)
        s = None if state is None else tensors(*state, dtype=f32)
        B.sol_attn3d_forward_linear(p, x, x, x, tensors(tokens, 4, 64), None, tensors(decay, dtype=f32), 1.0, s, None, None)

    call()
    call(q=(10, 256))                                                   # the same memory: fine
    call(q=(1, 10, 4, 64), state=(1, 4, 64, 64))
    assert calls == ["sol_attn3d_forward_linear"] * 3
    for bad in (dict(q=(10, 2, 128), decay=2), dict(decay=3), dict(q=(10, 2, 128), state=(1, 2, 128, 128)), dict(state=(2, 4, 64, 64)),
                dict(q=(9, 4, 64)), dict(tokens=9), dict(q=(10, 3, 64), decay=3)):
        with pytest.raises(ValueError):
            call(**bad)
    x = tensors(10, 4, 64)
    with pytest.raises(ValueError):
        B.sol_attn3d_forward_linear(p, x, x, x, tensors(10, 4, 64), tensors(9, dtype=torch.uint8), tensors(4, dtype=f32), 1.0)
    assert len(calls) == 3
    B.sol_attn3d_destroy(p)


def test_differential_weights_and_masks_are_the_plans(calls):
    p = B.sol_attn3d_plan_ex([(10, 0, 1, 1)], 8, 64, (16, 24, 24))

    def call(pairs=4, q=(10, 8, 64), tokens=10, mask=10, want=10):
        vec = tensors(64, dtype=torch.float32) if pairs is None else tensors(pairs, 64, dtype=torch.float32)
        w = B.sol_attn3d_diff_weights(vec, vec, vec, vec, 0.5, tensors(128, dtype=torch.float32))
        x = tensors(*q)
        B.sol_attn3d_forward_diff(p, x, x, x, tensors(tokens, 8, 64), tensors(mask, dtype=torch.uint8), w, tensors(want, dtype=torch.uint8))

    call()
    call(pairs=None)
    call(q=(10, 512))
    assert calls == ["sol_attn3d_forward_diff"] * 3
    for bad in (dict(q=(10, 4, 128), pairs=2), dict(pairs=8), dict(q=(9, 8, 64)), dict(tokens=9), dict(mask=9), dict(want=9)):
        with pytest.raises(ValueError):
            call(**bad)
    assert len(calls) == 3
    B.sol_attn3d_destroy(p)
