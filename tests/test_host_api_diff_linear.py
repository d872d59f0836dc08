"""CPU tests of the differential / linear attention entry points: what they refuse before anything is enqueued."""
import ctypes

import pytest
import torch

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


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the call would go on to use the made-up pointers")
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


def test_infinite_eps_and_capacities_beyond_32_bits_are_refused():
    lib = B._lib()
    p = B.sol_attn3d_plan(1, 4, 64, 4, 8, 8, 0, (16, 24, 24))
    w = _weights(eps=float("inf"))
    assert lib.sol_attn3d_forward_diff(p, 16, 32, 48, 64, None, None, ctypes.byref(w), None) == B.ERR_INVALID_ARG
    B.sol_attn3d_destroy(p)
    w = _weights()
    for capacity in (2 ** 31, 2 ** 40, 2 ** 62):
        c = B._KvCache(ctypes.sizeof(B._KvCache), 32, 48, (0, 0, 0), (0, 0, 0), 3, capacity, None, 0)
        assert lib.sol_attn3d_diff_step(16, _s2(), ctypes.byref(c), 4, None, 64, _s2(), 3, 4, 64, ctypes.byref(w), None, 0,
                                        None) == B.ERR_UNSUPPORTED_SHAPE
        assert B.sol_attn3d_diff_step_workspace_bytes(3, 4, 64, capacity) == 0
    assert B.sol_attn3d_diff_step_workspace_bytes(3, 4, 64, 2 ** 31 - 1) > 0


def _s2(a=0, b=0):
    return (ctypes.c_int64 * 2)(a, b)


def test_diff_step_refusals():
    lib = B._lib()
    w = _weights()

    def call(q=16, lens=4, slots=None, out=64, batch=3, heads=4, head_dim=64, ws=None, nbytes=0, w=w, q_st=(0, 0), **kw):
        c = B._KvCache(ctypes.sizeof(B._KvCache), 32, 48, (0, 0, 0), (0, 0, 0), 3, 4096, None, 0)
        for k, v in kw.items():
            setattr(c, k, (ctypes.c_int64 * 3)(*v) if k.endswith("k_strides") else v)
        return lib.sol_attn3d_diff_step(q, _s2(*q_st), ctypes.byref(c), lens, slots, out, _s2(), batch, heads, head_dim,
                                        ctypes.byref(w), ws, nbytes, None)

    need = B.sol_attn3d_diff_step_workspace_bytes(3, 4, 64, 4096)
    assert need > 0 and need % 256 == 0
    assert call() == B.ERR_NO_WORKSPACE                                # everything else is in order
    assert call(ws=256, nbytes=need - 1) == B.ERR_NO_WORKSPACE
    assert call(ws=128, nbytes=need) == B.ERR_NO_WORKSPACE
    assert call(batch=0, q=None, out=None, lens=None) == 0             # nothing to do
    for bad in (dict(q=None), dict(q=8), dict(out=16), dict(out=None), dict(lens=None), dict(lens=6), dict(slots=2), dict(k=None),
                dict(v=40), dict(batch=-1), dict(n_slots=-1), dict(capacity=-1), dict(size=8), dict(w=_weights(gain=4))):
        assert call(**bad) == B.ERR_INVALID_ARG, bad
    for bad in (dict(head_dim=128), dict(heads=3), dict(q_st=(257, 64)), dict(k_strides=(0, 260, 64)), dict(k_strides=(-8, 0, 0)),
                dict(mask_slot_stride=-1), dict(batch=2 ** 30, heads=8)):
        assert call(**bad) == B.ERR_UNSUPPORTED_SHAPE, bad
    assert B.sol_attn3d_diff_step_workspace_bytes(3, 3, 64, 4096) == 0
    assert B.sol_attn3d_diff_step_workspace_bytes(2000, 40, 64, 4096) == 0         # enough streams: no split


def test_linear_step_refusals():
    lib = B._lib()

    def call(q=16, k=32, v=48, out=64, st=(0, 0), batch=2, heads=4, head_dim=64, decay=4, scale=1.0, a=16, b=16, n_slots=2, slots=4):
        return lib.sol_attn3d_linear_step(q, k, v, out, _s2(), _s2(*st), _s2(), _s2(), batch, heads, head_dim, decay,
                                          scale, a, b, n_slots, slots, None)

    assert call(batch=0, q=None) == 0
    for bad in (dict(q=None), dict(v=8), dict(out=32), dict(out=None), dict(decay=None), dict(decay=2), dict(scale=float("nan")),
                dict(a=None), dict(b=8), dict(slots=6), dict(slots=None, n_slots=1), dict(batch=-1), dict(heads=0)):
        assert call(**bad) == B.ERR_INVALID_ARG, bad
    for bad in (dict(head_dim=96), dict(st=(257, 64)), dict(st=(-256, 64)), dict(batch=2 ** 30), dict(heads=70000)):
        assert call(**bad) == B.ERR_UNSUPPORTED_SHAPE, bad


def test_forward_linear_refusals_and_scratch_size():
    lib = B._lib()
    p = B.sol_attn3d_plan(1, 4, 64, 4, 8, 8, 0, (16, 24, 24))

    def call(plan=p, q=16, k=32, v=48, out=64, decay=4, scale=1.0, a=None, b=None):
        return lib.sol_attn3d_forward_linear(plan, q, k, v, out, None, decay, scale, a, b, None, 0, None)

    assert call() == B.ERR_NO_WORKSPACE                                # no workspace bound; everything else is in order
    for bad in (dict(plan=None), dict(q=None), dict(k=8), dict(out=16), dict(out=None), dict(decay=None), dict(decay=6),
                dict(scale=float("inf")), dict(a=8), dict(b=24)):
        assert call(**bad) == B.ERR_INVALID_ARG, bad
    assert B.sol_attn3d_linear_workspace_bytes(p) == 0                 # two tiles: one piece per head
    B.sol_attn3d_destroy(p)
    # a long sequence with few heads is cut; its scratch holds a state per piece with a successor and per (sequence, head)
    p = B.sol_attn3d_plan_ex([(256, 5, 30, 20)], 2, 128, (32, 48, 48))
    n = B.sol_attn3d_linear_workspace_bytes(p)
    assert n % (128 * 128 * 4) == 0 and n // (128 * 128 * 4) > 4
    B.sol_attn3d_destroy(p)


def test_expanded_tensors_are_refused():
    """0 stands for the dense stride at the C entry, so an expanded axis (torch stride 0) must not get there."""
    dense = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    assert list(B._row_strides(dense, 64)) == [256, 64]
    assert list(B._row_strides(dense[:1].expand(1, 4, 64), 64)) == [256, 64]      # an axis of one: any stride will do
    for bad in (dense[:1].expand(3, 4, 64), dense[:, :1].expand(3, 4, 64)):
        with pytest.raises(ValueError):
            B._row_strides(bad, 64)
    cache = torch.zeros(2, 5, 4, 64, dtype=torch.bfloat16)
    assert list(B._cache_strides(cache, cache.shape)) == [1280, 256, 64]
    for bad in (cache[:1].expand(2, 5, 4, 64), cache[:, :1].expand(2, 5, 4, 64), cache[:, :, :1].expand(2, 5, 4, 64)):
        with pytest.raises(ValueError):
            B._cache_strides(bad, cache.shape)


def test_first_questions_about_one_plan_from_several_threads_agree():
    """The cutting of sequences is planned once per plan, whoever asks first."""
    import threading
    lib = B._lib()
    for _ in range(20):
        p = B.sol_attn3d_plan_ex([(256, 5, 30, 20), (256, 16, 30, 52)], 20, 128, (32, 48, 48))
        start, got = threading.Barrier(4), []

        def ask():
            start.wait()
            got.append(lib.sol_attn3d_linear_workspace_bytes(p))     # ctypes releases the interpreter lock

        threads = [threading.Thread(target=ask) for _ in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert len(set(got)) == 1 and got[0] == B.sol_attn3d_linear_workspace_bytes(p)
        B.sol_attn3d_destroy(p)
