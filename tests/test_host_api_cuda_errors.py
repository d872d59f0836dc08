"""A CUDA error of a call without a plan can be asked for afterwards, on the thread that made the call."""
import ctypes
import threading

import pytest
import torch

from paper_2609_35110_b200 import binding as B
from paper_2609_35110_b200 import build as build_mod

I2 = ctypes.c_int64 * 2


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build_mod.build_library()


def calls():
    """Every call without a plan, with arguments that are in order (addresses of nothing: they fail before a kernel could look)."""
    lib, z = B._lib(), I2(0, 0)
    pool = B._PagedCache(ctypes.sizeof(B._PagedCache), 2, 64, 2, 64, 16, 32, (0, 0, 0, 0), (0, 0, 0, 0), 100, 64, 128, 192, 5, 10)
    states = B._Context(ctypes.sizeof(B._Context), 2, 64, 16, 32, (0, 0), (0, 0), 100, 64, 128, 77, None)
    cache, context = ctypes.byref(pool), ctypes.byref(states)
    book = lib.sol_attn3d_cache_workspace_bytes(cache, 1)
    dst = (ctypes.c_void_p * 2)(256, 512)
    return {
        "reserve": lambda: lib.sol_attn3d_cache_reserve(cache, 1, 64, 64, None, None),
        "fork": lambda: lib.sol_attn3d_cache_fork(cache, 1, 64, 64, None, 256, book, None),
        "compact": lambda: lib.sol_attn3d_cache_compact(cache, 1, 64, 64, 10, None, 256, book, None),
        "free": lambda: lib.sol_attn3d_cache_free(cache, 1, 64, None, None),
        "copy_pages": lambda: lib.sol_attn3d_cache_copy_pages(cache, 1, 64, 64, None),
        "paged_step": lambda: lib.sol_attn3d_paged_step(16, z, cache, 0, None, 32, z, 1, 4, None, 0, 256, 1 << 30, None),
        "cross_step": lambda: lib.sol_attn3d_cross_step(16, z, context, 32, z, 1, 4, None, 0, None),
        "linear_step": lambda: lib.sol_attn3d_linear_step(16, 32, 48, 64, z, z, z, z, 1, 4, 64, 80, 1.0, None, None, 0, 96, None),
        "pack": lambda: lib.sol_attn3d_exchange_pack_qkv(16, 32, 48, z, z, z, 4, 4, 64, 2, 0, 0, dst, 0, None),
    }


@pytest.mark.skipif(torch.cuda.is_available(), reason="the error is that there is no device")
@pytest.mark.parametrize("name", ["reserve", "fork", "compact", "free", "copy_pages", "paged_step", "cross_step", "linear_step", "pack"])
def test_the_code_is_kept(name):
    assert B.sol_attn3d_last_cuda_error(None) >= 0
    seen = []

    def run():
        seen.append(B.sol_attn3d_last_cuda_error(None))
        assert calls()[name]() == B.ERR_CUDA
        seen.append(B.sol_attn3d_last_cuda_error(None))
        assert B._lib().sol_attn3d_cache_free(None, 1, 64, None, None) == B.ERR_INVALID_ARG
        seen.append(B.sol_attn3d_last_cuda_error(None))                 # (a refusal is no CUDA error)

    before = B.sol_attn3d_last_cuda_error(None)
    worker = threading.Thread(target=run)
    worker.start()
    worker.join()
    assert seen[0] == 0 and seen[1] > 0 and seen[2] == seen[1]
    assert B.sol_attn3d_last_cuda_error(None) == before                 # another thread's


def test_a_plan_keeps_its_own():
    p = B.sol_attn3d_plan(1, 4, 64, 1, 4, 8, 0, (16, 24, 24))
    assert B.sol_attn3d_last_cuda_error(p) == 0
    B.sol_attn3d_destroy(p)
