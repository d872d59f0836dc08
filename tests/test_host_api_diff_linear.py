"""CPU tests of the differential / linear attention entry points: what they refuse before anything is enqueued."""
import ctypes

import pytest

from paper_2609_35110_b200 import binding as B
from paper_2609_35110_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build_mod.build_library()
    return B._lib()


def _weights(**kw):
    w = B._DiffWeights(ctypes.sizeof(B._DiffWeights), 0.5, 64, 64, 64, 64, 0, 128, 1e-5)
    for k, v in kw.items():
        setattr(w, k, v)
    return w


def test_forward_diff_refusals():
    lib = B._lib()
    p = B.sol_attn3d_plan(1, 4, 64, 4, 8, 8, 0, (16, 24, 24))
    odd = B.sol_attn3d_plan(1, 3, 64, 4, 8, 8, 0, (16, 24, 24))
    wide = B.sol_attn3d_plan(1, 4, 128, 4, 8, 8, 0, (32, 48, 48))

    def call(plan=p, q=16, k=32, v=48, out=64, w=None, **kw):
        w = _weights(**kw) if w is None else w
        return lib.sol_attn3d_forward_diff(plan, q, k, v, out, None, None, ctypes.byref(w), None)

    assert call() == B.ERR_NO_WORKSPACE                               # everything else is in order
    assert call(gain=None) == B.ERR_NO_WORKSPACE
    assert call(lambda_pair_stride=64) == B.ERR_NO_WORKSPACE
    assert call(plan=odd) == B.ERR_UNSUPPORTED_SHAPE
    assert call(plan=wide) == B.ERR_UNSUPPORTED_SHAPE
    assert call(plan=None) == B.ERR_INVALID_ARG
    for bad in (dict(q=None), dict(out=None), dict(k=8), dict(out=16), dict(out=48), dict(size=4), dict(lambda_q1=None),
                dict(lambda_k2=66), dict(lambda_pair_stride=63), dict(lambda_pair_stride=-64), dict(gain=132), dict(eps=-1.0),
                dict(eps=float("nan")), dict(lambda_init=float("inf"))):
        assert call(**bad) == B.ERR_INVALID_ARG, bad
    assert lib.sol_attn3d_forward_diff(p, 16, 32, 48, 64, None, None, None, None) == B.ERR_INVALID_ARG
    assert B.sol_attn3d_last_launch_count(p) == 0
    for x in (p, odd, wide):
        B.sol_attn3d_destroy(x)


def test_differential_workspace_leaves_the_builtin_scratch_limit_alone():
    """The scratch of sol_attn3d_forward_noalloc counts what the plain forward uses: a plan just under 32 MiB without the
    differential attention's few bytes stays accepted (it is refused for the missing device, not for its size)."""
    lib = B._lib()
    rot = 2 * 64 * 2 * 2                                              # bytes of Q~ and K~ per token at 2 heads
    n = 32 * 2 ** 20 // rot
    while True:                                                       # the longest prefix-only plan whose dense part fits
        p = B.sol_attn3d_plan_ex([(n, 0, 1, 1)], 2, 64, (0, 0, 0))
        code = lib.sol_attn3d_forward_noalloc(p, 16, 32, 48, 64, None, None, None)
        total = B.sol_attn3d_workspace_bytes(p)
        B.sol_attn3d_destroy(p)
        if code != B.ERR_SCRATCH_LIMIT:
            break
        n -= 1
    assert total > 32 * 2 ** 20
