"""CPU tests of the entry points of streaming generation: what they refuse before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2609_35110_b200 import binding as B
from paper_2609_35110_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build_mod.build_library()
    return B._lib()


def cache(**kw):
    c = B._PagedCache(ctypes.sizeof(B._PagedCache), 2, 64, 2, 64, 16, 32, (0, 0, 0, 0), (0, 0, 0, 0), 100, 64, 128, 192, 5, 10)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def context(**kw):
    c = B._Context(ctypes.sizeof(B._Context), 2, 64, 16, 32, (0, 0), (0, 0), 100, 64, 128, 77, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


I2, I4 = ctypes.c_int64 * 2, ctypes.c_int64 * 4
INVALID = [dict(size=4), dict(n_layers=0), dict(page_size=0), dict(kv_heads=0), dict(head_dim=0), dict(n_pages=0), dict(n_streams=0),
           dict(table_width=0), dict(k=None), dict(v=None), dict(k=8), dict(table=None), dict(lens=None), dict(table=66), dict(refs=2)]
UNSUPPORTED = [dict(head_dim=96), dict(page_size=24), dict(page_size=4112), dict(n_pages=1 << 26), dict(table_width=1 << 26), dict(kv_heads=65536),
               dict(k_strides=I4(0, 0, 4, 0)), dict(v_strides=I4(0, 0, 0, -64)), dict(k_strides=I4(-8, 0, 0, 0)), dict(v_strides=I4(0, 12, 0, 0))]


def test_cache_is_checked_by_every_call():
    lib = B._lib()
    p = B.sol_attn3d_plan(1, 4, 64, 1, 4, 8, 0, (16, 24, 24))
    z = I2(0, 0)
    calls = [
        lambda c: lib.sol_attn3d_cache_reserve(c, 1, 64, 64, None, None),
        lambda c: lib.sol_attn3d_cache_fork(c, 1, 64, 64, None, None, 0, None),
        lambda c: lib.sol_attn3d_cache_compact(c, 1, 64, 64, 10, None, None, 0, None),
        lambda c: lib.sol_attn3d_cache_free(c, 0, 64, None, None),
        lambda c: lib.sol_attn3d_cache_copy_pages(c, 0, 64, 64, None),
        lambda c: lib.sol_attn3d_cache_append(p, 16, 16, 16, z, z, 32, c, 0, None, None, None, None, 0.0, None),
        lambda c: lib.sol_attn3d_forward_paged(p, 16, c, 0, 32, None, None, 0, 0, None, 0, None),
        lambda c: lib.sol_attn3d_paged_step(16, z, c, 0, None, 32, z, 1, 4, None, 0, None, 0, None),
    ]
    for call in calls:
        for bad in INVALID:
            assert call(cache(**bad)) == B.ERR_INVALID_ARG, bad
        for bad in UNSUPPORTED:
            assert call(cache(**bad)) == B.ERR_UNSUPPORTED_SHAPE, bad
        assert call(None) == B.ERR_INVALID_ARG
    for bad in INVALID + UNSUPPORTED:
        assert lib.sol_attn3d_cache_workspace_bytes(cache(**bad), 3) == 0
        assert lib.sol_attn3d_paged_workspace_bytes(p, cache(**bad)) == 0
        assert lib.sol_attn3d_paged_step_workspace_bytes(cache(**bad), 1, 4) == 0
    B.sol_attn3d_destroy(p)


def test_bookkeeping_refusals():
    lib = B._lib()
    need = lib.sol_attn3d_cache_workspace_bytes(cache(), 3)
    assert need >= 3 * 640 * 8 and lib.sol_attn3d_cache_workspace_bytes(cache(), 0) == 0 and lib.sol_attn3d_cache_workspace_bytes(cache(), 2049) == 0
    fork = lambda n=3, a=64, b=64, st=None, ws=256, size=need, c=None: lib.sol_attn3d_cache_fork(c or cache(), n, a, b, st, ws, size, None)
    thin = lambda n=3, a=64, keep=64, width=10, st=None, ws=256, size=need, c=None: lib.sol_attn3d_cache_compact(c or cache(), n, a, keep, width, st, ws, size, None)
    grow = lambda n=3, a=64, b=64, st=None, c=None: lib.sol_attn3d_cache_reserve(c or cache(), n, a, b, st, None)
    close = lambda n=3, a=64, st=None, c=None: lib.sol_attn3d_cache_free(c or cache(), n, a, st, None)
    for f in (fork, thin, grow, close):
        assert f(n=0) == B.OK                                           # nothing to do
        assert f(n=-1) == B.ERR_INVALID_ARG and f(a=None) == B.ERR_INVALID_ARG and f(a=65) == B.ERR_INVALID_ARG and f(st=66) == B.ERR_INVALID_ARG
        assert f(n=2049) == B.ERR_UNSUPPORTED_SHAPE
        assert f(c=cache(refs=None)) == B.ERR_INVALID_ARG
    for f in (fork, grow):
        assert f(b=None) == B.ERR_INVALID_ARG and f(b=66) == B.ERR_INVALID_ARG
    for f in (fork, thin):
        assert f(ws=None) == B.ERR_NO_WORKSPACE and f(ws=128) == B.ERR_NO_WORKSPACE and f(size=need - 1) == B.ERR_NO_WORKSPACE
    assert thin(keep=None) == B.ERR_INVALID_ARG and thin(width=0) == B.ERR_INVALID_ARG
    copy = lambda n, a, b: lib.sol_attn3d_cache_copy_pages(cache(), n, a, b, None)
    assert copy(0, None, None) == B.OK and copy(-1, 64, 64) == B.ERR_INVALID_ARG and copy(2, None, 64) == B.ERR_INVALID_ARG
    assert copy(2, 64, 65) == B.ERR_INVALID_ARG and copy((1 << 20) + 1, 64, 64) == B.ERR_UNSUPPORTED_SHAPE


def test_append_refusals():
    lib = B._lib()
    p = B.sol_attn3d_plan(1, 4, 64, 1, 4, 8, 0, (16, 24, 24))
    wide = B.sol_attn3d_plan(1, 4, 128, 1, 4, 8, 0, (32, 48, 48))

    def call(plan=p, q=16, k=32, v=48, ks=I2(0, 0), vs=I2(0, 0), out=64, layer=0, streams=None, pos0=None, qg=None, kg=None, eps=0.0):
        return lib.sol_attn3d_cache_append(plan, q, k, v, ks, vs, out, cache(), layer, streams, pos0, qg, kg, eps, None)

    assert call() == B.ERR_NO_WORKSPACE                                 # everything else is in order
    assert call(q=None, out=None) == B.ERR_NO_WORKSPACE
    for bad in (dict(plan=None), dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(ks=None), dict(vs=None), dict(out=16), dict(out=32), dict(out=48),
                dict(q=8), dict(v=8), dict(qg=8), dict(kg=24), dict(streams=2), dict(pos0=6), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(layer=-1), dict(layer=2)):
        assert call(**bad) == B.ERR_INVALID_ARG, bad
    for bad in (dict(plan=wide), dict(ks=I2(4, 0)), dict(vs=I2(0, -8))):
        assert call(**bad) == B.ERR_UNSUPPORTED_SHAPE, bad
    for x in (p, wide):
        B.sol_attn3d_destroy(x)


def test_forward_refusals():
    lib = B._lib()
    p = B.sol_attn3d_plan(1, 4, 64, 1, 4, 8, 0, (16, 24, 24))
    odd = B.sol_attn3d_plan(1, 3, 64, 1, 4, 8, 0, (16, 24, 24))
    wide = B.sol_attn3d_plan(1, 4, 128, 1, 4, 8, 0, (32, 48, 48))

    def paged(plan=p, q=16, layer=1, out=32, streams=None, mask=None, width=0, causal=0):
        return lib.sol_attn3d_forward_paged(plan, q, cache(), layer, out, streams, mask, width, causal, None, 0, None)

    def cross(plan=p, q=16, out=32, **kw):
        return lib.sol_attn3d_forward_cross(plan, q, context(**kw), out, None, 0, None)

    for f in (paged, cross):
        assert f() == B.ERR_NO_WORKSPACE                                # the plan has none
        for bad in (dict(plan=None), dict(q=None), dict(out=None), dict(q=8), dict(out=8), dict(out=16)):
            assert f(**bad) == B.ERR_INVALID_ARG, bad
        assert f(plan=odd) == B.ERR_UNSUPPORTED_SHAPE and f(plan=wide) == B.ERR_UNSUPPORTED_SHAPE
    for bad in (dict(layer=2), dict(layer=-1), dict(streams=2), dict(mask=1, width=0), dict(causal=-1)):
        assert paged(**bad) == B.ERR_INVALID_ARG, bad
    bad_contexts = [dict(size=1), dict(kv_heads=0), dict(head_dim=0), dict(total_rows=-1), dict(max_len=-1), dict(begins=None), dict(lens=None), dict(begins=2), dict(k=None),
                    dict(v=None), dict(k=8)]
    odd_contexts = [dict(head_dim=32), dict(kv_heads=65536), dict(total_rows=1 << 31), dict(k_strides=I2(0, 4)), dict(v_strides=I2(-64, 0))]
    step = lambda **kw: lib.sol_attn3d_cross_step(16, I2(0, 0), context(**kw), 32, I2(0, 0), 1, 4, None, 0, None)
    for f in (cross, step):
        for bad in bad_contexts:
            assert f(**bad) == B.ERR_INVALID_ARG, bad
        for bad in odd_contexts:
            assert f(**bad) == B.ERR_UNSUPPORTED_SHAPE, bad
    for bad in bad_contexts + odd_contexts:
        assert lib.sol_attn3d_cross_workspace_bytes(p, context(**bad)) == 0 and lib.sol_attn3d_cross_step_workspace_bytes(context(**bad), 1, 4) == 0
    assert B.sol_attn3d_last_launch_count(p) == 0
    for x in (p, odd, wide):
        B.sol_attn3d_destroy(x)


def test_step_refusals():
    lib = B._lib()
    z = I2(0, 0)

    def paged(q=16, qs=z, layer=0, streams=None, out=32, os=z, batch=1, heads=4, mask=None, width=0, c=None, ws=None, size=0):
        return lib.sol_attn3d_paged_step(q, qs, c or cache(), layer, streams, out, os, batch, heads, mask, width, ws, size, None)

    def cross(q=16, qs=z, out=32, os=z, batch=1, heads=4, c=None, ws=None, size=0):
        return lib.sol_attn3d_cross_step(q, qs, c or context(), out, os, batch, heads, ws, size, None)

    for f in (paged, cross):
        assert f(batch=0) == B.OK
        for bad in (dict(q=None), dict(out=None), dict(q=8), dict(out=8), dict(out=16), dict(qs=None), dict(os=None), dict(batch=-1), dict(heads=0)):
            assert f(**bad) == B.ERR_INVALID_ARG, bad
        for bad in (dict(heads=3), dict(heads=65536), dict(qs=I2(4, 0)), dict(os=I2(0, -64)), dict(batch=1 << 30, heads=16)):
            assert f(**bad) == B.ERR_UNSUPPORTED_SHAPE, bad
    long_cache, long_context = cache(table_width=1 << 20), context(total_rows=1 << 20, max_len=1 << 20)
    need = lib.sol_attn3d_paged_step_workspace_bytes(long_cache, 1, 4)
    assert need > 0 and need == lib.sol_attn3d_cross_step_workspace_bytes(long_context, 1, 4)
    for f, c in ((paged, long_cache), (cross, long_context)):
        for bad in (dict(), dict(ws=256, size=need - 1), dict(ws=128, size=need)):
            assert f(c=c, **bad) == B.ERR_NO_WORKSPACE, bad
    assert paged(layer=2) == B.ERR_INVALID_ARG and paged(streams=2) == B.ERR_INVALID_ARG and paged(mask=1) == B.ERR_INVALID_ARG


def test_binding_refuses_what_the_library_cannot_see():
    """Types and shapes; on a machine without a device every tensor is refused for living on the CPU."""
    x = torch.zeros(1, 2, 16, 1, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.sol_attn3d_paged_cache(x, x, torch.zeros(2, 3, dtype=torch.int32), i)
    with pytest.raises(ValueError):
        B.sol_attn3d_context(x[0, 0], x[0, 0], i, i, 5)
