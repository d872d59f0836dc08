"""ctypes binding of the C-ABI library, one Python function per exported call.

Argument marshalling only: every step of the attention path runs in the CUDA
kernels behind ``libsol_attn3d.so``.  PyTorch appears here only as the owner
of device memory and streams.  There is no CPU fallback: loading fails loudly
if the library has not been built, and device calls fail on a machine without
a B200.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SOL_ATTN3D_LIB") or os.path.join(_HERE, "libsol_attn3d.so")


class SolAttn3dError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = _lib().sol_attn3d_strerror(code).decode() if _LIB is not None else "?"
        super().__init__(f"{where}: {msg} (code {code})")


class sol_attn3d_desc(ctypes.Structure):
    _fields_ = [
        ("size", ctypes.c_uint32),
        ("n_seqs", ctypes.c_int32),
        ("grids", ctypes.POINTER(ctypes.c_int32)),
        ("text_lens", ctypes.POINTER(ctypes.c_int32)),
        ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("rope_dims", ctypes.c_int32 * 3),
        ("theta", ctypes.c_double),
        ("q_strides", ctypes.c_int64 * 2),
        ("k_strides", ctypes.c_int64 * 2),
        ("v_strides", ctypes.c_int64 * 2),
        ("out_strides", ctypes.c_int64 * 2),
    ]


class _DiffWeights(ctypes.Structure):
    _fields_ = [
        ("size", ctypes.c_uint32),
        ("lambda_init", ctypes.c_float),
        ("lambda_q1", ctypes.c_void_p),
        ("lambda_k1", ctypes.c_void_p),
        ("lambda_q2", ctypes.c_void_p),
        ("lambda_k2", ctypes.c_void_p),
        ("lambda_pair_stride", ctypes.c_int64),
        ("gain", ctypes.c_void_p),
        ("eps", ctypes.c_float),
    ]


class _KvCache(ctypes.Structure):
    _fields_ = [
        ("size", ctypes.c_uint32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_strides", ctypes.c_int64 * 3),
        ("v_strides", ctypes.c_int64 * 3),
        ("n_slots", ctypes.c_int64),
        ("capacity", ctypes.c_int64),
        ("key_mask", ctypes.c_void_p),
        ("mask_slot_stride", ctypes.c_int64),
    ]


class _PagedCache(ctypes.Structure):
    _fields_ = [
        ("size", ctypes.c_uint32),
        ("n_layers", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_strides", ctypes.c_int64 * 4),
        ("v_strides", ctypes.c_int64 * 4),
        ("n_pages", ctypes.c_int64),
        ("table", ctypes.c_void_p),
        ("lens", ctypes.c_void_p),
        ("refs", ctypes.c_void_p),
        ("n_streams", ctypes.c_int64),
        ("table_width", ctypes.c_int64),
    ]


class _Context(ctypes.Structure):
    _fields_ = [
        ("size", ctypes.c_uint32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_strides", ctypes.c_int64 * 2),
        ("v_strides", ctypes.c_int64 * 2),
        ("total_rows", ctypes.c_int64),
        ("begins", ctypes.c_void_p),
        ("lens", ctypes.c_void_p),
        ("max_len", ctypes.c_int64),
        ("key_mask", ctypes.c_void_p),
    ]


_KV_CACHE_SIZE = ctypes.sizeof(_KvCache)


# error codes (mirror include/sol_attn3d.h)
OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED_SHAPE = -2
ERR_NO_WORKSPACE = -3
ERR_NO_DEVICE = -4
ERR_UNSUPPORTED_ARCH = -5
ERR_CUDA = -6
ERR_DEVICE_TIMEOUT = -7
ERR_NO_MEMORY = -8
ERR_SCRATCH_LIMIT = -9
ERR_DEVICE_ASSERT = -10

# what the bookkeeping calls of a paged cache say of each request
CACHE_OK = 0
CACHE_BAD_STREAM = 1
CACHE_NO_ROOM = 2
CACHE_NO_PAGES = 3
CACHE_NOT_EMPTY = 4

_LIB = None


def _lib():
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2609_35110_b200.build` "
            "(there is no CPU fallback for the attention path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    lib.sol_attn3d_plan.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
    lib.sol_attn3d_plan.restype = i32
    lib.sol_attn3d_plan_ex.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(sol_attn3d_desc)]
    lib.sol_attn3d_plan_ex.restype = i32
    lib.sol_attn3d_cu_seqlens.argtypes = [vp, ctypes.POINTER(ctypes.POINTER(i64)), ctypes.POINTER(i32)]
    lib.sol_attn3d_cu_seqlens.restype = i32
    lib.sol_attn3d_workspace_bytes.argtypes = [vp]
    lib.sol_attn3d_workspace_bytes.restype = ctypes.c_size_t
    lib.sol_attn3d_set_workspace.argtypes = [vp, vp, ctypes.c_size_t]
    lib.sol_attn3d_set_workspace.restype = i32
    lib.sol_attn3d_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.sol_attn3d_forward.restype = i32
    lib.sol_attn3d_forward_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.sol_attn3d_forward_noalloc.restype = i32
    lib.sol_attn3d_forward_qknorm.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp]
    lib.sol_attn3d_forward_qknorm.restype = i32
    lib.sol_attn3d_qknorm_rope.argtypes = [vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp]
    lib.sol_attn3d_qknorm_rope.restype = i32
    lib.sol_attn3d_forward_rect.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.sol_attn3d_forward_rect.restype = i32
    lib.sol_attn3d_forward_e4m3.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.sol_attn3d_forward_e4m3.restype = i32
    lib.sol_attn3d_forward_int8.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.sol_attn3d_forward_int8.restype = i32
    lib.sol_attn3d_forward_qkv_int8.argtypes = [vp, vp, vp, vp, vp, i32, vp]
    lib.sol_attn3d_forward_qkv_int8.restype = i32
    lib.sol_attn3d_forward_scatter.argtypes = [vp, vp, vp, vp, vp, i32, ctypes.POINTER(vp), ctypes.POINTER(i64), i32, i32,
                                               i32, vp]
    lib.sol_attn3d_forward_scatter.restype = i32
    lib.sol_attn3d_exchange_pack_qkv.argtypes = [vp, vp, vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64),
                                                 i64, i32, i32, i32, i32, i32, ctypes.POINTER(vp), i64, vp]
    lib.sol_attn3d_exchange_pack_qkv.restype = i32
    lib.sol_attn3d_exchange_merge_heads.argtypes = [vp, vp, i64, i32, i32, i32, i64, i64, vp]
    lib.sol_attn3d_exchange_merge_heads.restype = i32
    lib.sol_attn3d_exchange_record_bytes.argtypes = [i32, i32]
    lib.sol_attn3d_exchange_record_bytes.restype = ctypes.c_size_t
    lib.sol_attn3d_exchange_pack_qkv_int8.argtypes = lib.sol_attn3d_exchange_pack_qkv.argtypes
    lib.sol_attn3d_exchange_pack_qkv_int8.restype = i32
    lib.sol_attn3d_exchange_unpack_qkv_int8.argtypes = [vp, vp, i64, i32, i32, vp]
    lib.sol_attn3d_exchange_unpack_qkv_int8.restype = i32
    lib.sol_attn3d_exchange_quantize_out_int8.argtypes = [vp, ctypes.POINTER(i64), i64, i32, i32, vp, vp]
    lib.sol_attn3d_exchange_quantize_out_int8.restype = i32
    lib.sol_attn3d_exchange_dequantize_out_int8.argtypes = [vp, vp, i64, i32, i32, vp]
    lib.sol_attn3d_exchange_dequantize_out_int8.restype = i32
    lib.sol_attn3d_host_staging_bytes.argtypes = [vp]
    lib.sol_attn3d_host_staging_bytes.restype = ctypes.c_size_t
    lib.sol_attn3d_forward_host.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, i32, vp]
    lib.sol_attn3d_forward_host.restype = i32
    lib.sol_attn3d_sparse_workspace_bytes.argtypes = [vp]
    lib.sol_attn3d_sparse_workspace_bytes.restype = ctypes.c_size_t
    lib.sol_attn3d_forward_sparse.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, ctypes.c_size_t, vp]
    lib.sol_attn3d_forward_sparse.restype = i32
    lib.sol_attn3d_sparse_stats.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(ctypes.c_longlong)]
    lib.sol_attn3d_sparse_stats.restype = i32
    lib.sol_attn3d_sparse_selection.argtypes = [vp, vp, i32, i32, i32, ctypes.POINTER(i32), i32, ctypes.POINTER(i32)]
    lib.sol_attn3d_sparse_selection.restype = i32
    lib.sol_attn3d_plan_dims.argtypes = [vp, ctypes.POINTER(i64)]
    lib.sol_attn3d_plan_dims.restype = i32
    lib.sol_attn3d_forward_diff.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(_DiffWeights), vp]
    lib.sol_attn3d_forward_diff.restype = i32
    p64 = ctypes.POINTER(i64)
    lib.sol_attn3d_diff_step_workspace_bytes.argtypes = [i32, i32, i32, i64]
    lib.sol_attn3d_diff_step_workspace_bytes.restype = ctypes.c_size_t
    lib.sol_attn3d_diff_step.argtypes = [vp, p64, ctypes.POINTER(_KvCache), vp, vp, vp, p64, i32, i32, i32,
                                         ctypes.POINTER(_DiffWeights), vp, ctypes.c_size_t, vp]
    lib.sol_attn3d_diff_step.restype = i32
    lib.sol_attn3d_linear_workspace_bytes.argtypes = [vp]
    lib.sol_attn3d_linear_workspace_bytes.restype = ctypes.c_size_t
    lib.sol_attn3d_forward_linear.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp]
    lib.sol_attn3d_forward_linear.restype = i32
    lib.sol_attn3d_linear_step.argtypes = [vp, vp, vp, vp, p64, p64, p64, p64, i32, i32, i32, vp, ctypes.c_float, vp, vp, i64,
                                           vp, vp]
    lib.sol_attn3d_linear_step.restype = i32
    cache, context, size = ctypes.POINTER(_PagedCache), ctypes.POINTER(_Context), ctypes.c_size_t
    lib.sol_attn3d_cache_workspace_bytes.argtypes = [cache, i32]
    lib.sol_attn3d_cache_workspace_bytes.restype = size
    lib.sol_attn3d_cache_reserve.argtypes = [cache, i32, vp, vp, vp, vp]
    lib.sol_attn3d_cache_reserve.restype = i32
    lib.sol_attn3d_cache_fork.argtypes = [cache, i32, vp, vp, vp, vp, size, vp]
    lib.sol_attn3d_cache_fork.restype = i32
    lib.sol_attn3d_cache_compact.argtypes = [cache, i32, vp, vp, i64, vp, vp, size, vp]
    lib.sol_attn3d_cache_compact.restype = i32
    lib.sol_attn3d_cache_free.argtypes = [cache, i32, vp, vp, vp]
    lib.sol_attn3d_cache_free.restype = i32
    lib.sol_attn3d_cache_copy_pages.argtypes = [cache, i32, vp, vp, vp]
    lib.sol_attn3d_cache_copy_pages.restype = i32
    lib.sol_attn3d_cache_append.argtypes = [vp, vp, vp, vp, p64, p64, vp, cache, i32, vp, vp, vp, vp, ctypes.c_float, vp]
    lib.sol_attn3d_cache_append.restype = i32
    lib.sol_attn3d_paged_workspace_bytes.argtypes = [vp, cache]
    lib.sol_attn3d_paged_workspace_bytes.restype = size
    lib.sol_attn3d_forward_paged.argtypes = [vp, vp, cache, i32, vp, vp, vp, i64, i32, vp, size, vp]
    lib.sol_attn3d_forward_paged.restype = i32
    lib.sol_attn3d_paged_step_workspace_bytes.argtypes = [cache, i32, i32]
    lib.sol_attn3d_paged_step_workspace_bytes.restype = size
    lib.sol_attn3d_paged_step.argtypes = [vp, p64, cache, i32, vp, vp, p64, i32, i32, vp, i64, vp, size, vp]
    lib.sol_attn3d_paged_step.restype = i32
    lib.sol_attn3d_cross_workspace_bytes.argtypes = [vp, context]
    lib.sol_attn3d_cross_workspace_bytes.restype = size
    lib.sol_attn3d_forward_cross.argtypes = [vp, vp, context, vp, vp, size, vp]
    lib.sol_attn3d_forward_cross.restype = i32
    lib.sol_attn3d_cross_step_workspace_bytes.argtypes = [context, i32, i32]
    lib.sol_attn3d_cross_step_workspace_bytes.restype = size
    lib.sol_attn3d_cross_step.argtypes = [vp, p64, context, vp, p64, i32, i32, vp, size, vp]
    lib.sol_attn3d_cross_step.restype = i32
    lib.sol_attn3d_rope_qk.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.sol_attn3d_rope_qk.restype = i32
    lib.sol_attn3d_status.argtypes = [vp]
    lib.sol_attn3d_status.restype = i32
    lib.sol_attn3d_status_word.argtypes = [vp, ctypes.POINTER(ctypes.c_uint)]
    lib.sol_attn3d_status_word.restype = i32
    lib.sol_attn3d_debug_build.argtypes = []
    lib.sol_attn3d_debug_build.restype = i32
    lib.sol_attn3d_set_profiling.argtypes = [vp, i32]
    lib.sol_attn3d_set_profiling.restype = i32
    lib.sol_attn3d_last_forward_ms.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
    lib.sol_attn3d_last_forward_ms.restype = i32
    lib.sol_attn3d_last_launch_count.argtypes = [vp]
    lib.sol_attn3d_last_launch_count.restype = i32
    lib.sol_attn3d_softmax_rescale_count.argtypes = [vp, ctypes.POINTER(ctypes.c_ulonglong)]
    lib.sol_attn3d_softmax_rescale_count.restype = i32
    lib.sol_attn3d_last_cuda_error.argtypes = [vp]
    lib.sol_attn3d_last_cuda_error.restype = i32
    lib.sol_attn3d_strerror.argtypes = [i32]
    lib.sol_attn3d_strerror.restype = ctypes.c_char_p
    lib.sol_attn3d_destroy.argtypes = [vp]
    lib.sol_attn3d_destroy.restype = i32
    _LIB = lib
    return lib


def _check(code: int, where: str) -> None:
    if code != OK:
        raise SolAttn3dError(code, where)


# ----------------------------------------------------------------- 1:1 wrappers
class _Plan(ctypes.c_void_p):
    """A plan's handle; `dims` (what sol_attn3d_plan_dims answers) is kept with it once asked for, `device` (where its workspace is) once
    one is bound, `strides` (element strides of q and of out) from the start."""


def sol_attn3d_plan(B: int, heads: int, head_dim: int, T: int, H: int, W: int, text_len: int,
                    rope_dims: Sequence[int]) -> ctypes.c_void_p:
    h = _Plan()
    rd = (ctypes.c_int * 3)(*[int(x) for x in rope_dims])
    _check(_lib().sol_attn3d_plan(ctypes.byref(h), B, heads, head_dim, T, H, W, text_len, rd), "sol_attn3d_plan")
    h.strides = dict.fromkeys(("q", "out"), (heads * head_dim, head_dim, 1))
    return h


def sol_attn3d_plan_ex(seqs: Sequence[Tuple[int, int, int, int]], heads: int, head_dim: int,
                       rope_dims: Sequence[int], theta: float = 10000.0,
                       q_strides=(0, 0), k_strides=(0, 0), v_strides=(0, 0), out_strides=(0, 0)) -> ctypes.c_void_p:
    """seqs: [(text_len, T, H, W), ...]; strides are (token, head) element strides, 0 = contiguous."""
    n = len(seqs)
    grids = (ctypes.c_int32 * (3 * max(n, 1)))()
    lens = (ctypes.c_int32 * max(n, 1))()
    for i, (L, T, H, W) in enumerate(seqs):
        grids[3 * i], grids[3 * i + 1], grids[3 * i + 2] = T, H, W
        lens[i] = L
    d = sol_attn3d_desc()
    d.size = ctypes.sizeof(sol_attn3d_desc)
    d.n_seqs = n
    d.grids = ctypes.cast(grids, ctypes.POINTER(ctypes.c_int32))
    d.text_lens = ctypes.cast(lens, ctypes.POINTER(ctypes.c_int32))
    d.heads, d.head_dim = heads, head_dim
    for a in range(3):
        d.rope_dims[a] = int(rope_dims[a])
    d.theta = float(theta)
    for name, val in (("q_strides", q_strides), ("k_strides", k_strides), ("v_strides", v_strides),
                      ("out_strides", out_strides)):
        arr = getattr(d, name)
        arr[0], arr[1] = int(val[0]), int(val[1])
    h = _Plan()
    _check(_lib().sol_attn3d_plan_ex(ctypes.byref(h), ctypes.byref(d)), "sol_attn3d_plan_ex")
    h.strides = {name: (int(val[0]) or heads * head_dim, int(val[1]) or head_dim, 1) for name, val in (("q", q_strides), ("out", out_strides))}
    return h


def sol_attn3d_cu_seqlens(plan) -> list:
    p = ctypes.POINTER(ctypes.c_int64)()
    n = ctypes.c_int()
    _check(_lib().sol_attn3d_cu_seqlens(plan, ctypes.byref(p), ctypes.byref(n)), "sol_attn3d_cu_seqlens")
    return [int(p[i]) for i in range(n.value + 1)]


_I64x4 = ctypes.c_int64 * 4


def sol_attn3d_plan_dims(plan) -> Tuple[int, int, int, int]:
    """(sequences, heads, head_dim, total tokens)"""
    dims = _I64x4()
    _check(_lib().sol_attn3d_plan_dims(plan, dims), "sol_attn3d_plan_dims")
    return tuple(dims)


def sol_attn3d_workspace_bytes(plan) -> int:
    return int(_lib().sol_attn3d_workspace_bytes(plan))


def sol_attn3d_set_workspace(plan, workspace: torch.Tensor) -> None:
    _check(_lib().sol_attn3d_set_workspace(plan, workspace.data_ptr(), workspace.numel() * workspace.element_size()),
           "sol_attn3d_set_workspace")
    if isinstance(plan, _Plan):
        plan.device = workspace.get_device()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:                   # the raw handle: torch.cuda.current_stream() builds a Stream object every time
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def sol_attn3d_forward(plan, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       key_mask: Optional[torch.Tensor] = None, stream=None) -> None:
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    if key_mask is not None and (not key_mask.is_cuda or key_mask.dtype != torch.uint8 or not key_mask.is_contiguous()):
        raise ValueError("key_mask must be a contiguous CUDA uint8 tensor")
    _check(_lib().sol_attn3d_forward(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask), _stream(stream)),
           "sol_attn3d_forward")


def sol_attn3d_forward_noalloc(plan, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                               key_mask: Optional[torch.Tensor] = None, device_status: Optional[torch.Tensor] = None,
                               stream=None) -> None:
    """Forward without a caller workspace: the scratch is the 32 MiB array inside the library.

    For callers that may not allocate device memory (see include/sol_attn3d.h).  ``device_status`` is an
    optional CUDA int32 tensor with one element that receives the call's status word.  Calls on one
    device must not overlap on the GPU.
    """
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    if key_mask is not None and (not key_mask.is_cuda or key_mask.dtype != torch.uint8 or not key_mask.is_contiguous()):
        raise ValueError("key_mask must be a contiguous CUDA uint8 tensor")
    if device_status is not None and (not device_status.is_cuda or device_status.element_size() != 4):
        raise ValueError("device_status must be a CUDA tensor of 4-byte elements")
    _check(_lib().sol_attn3d_forward_noalloc(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask),
                                             _ptr(device_status), _stream(stream)), "sol_attn3d_forward_noalloc")


def sol_attn3d_forward_rect(plan, q, k, v, out, key_mask, query_mask: torch.Tensor, stream=None) -> None:
    """Rectangular forward: only rows with query_mask != 0 are computed and written; all tokens are keys."""
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    if not query_mask.is_cuda or query_mask.dtype != torch.uint8 or not query_mask.is_contiguous():
        raise ValueError("query_mask must be a contiguous CUDA uint8 tensor")
    _check(_lib().sol_attn3d_forward_rect(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask), _ptr(query_mask),
                                          _stream(stream)), "sol_attn3d_forward_rect")


def sol_attn3d_host_staging_bytes(plan) -> int:
    return int(_lib().sol_attn3d_host_staging_bytes(plan))


def sol_attn3d_forward_host(plan, q_host: torch.Tensor, k_host: torch.Tensor, v_host: torch.Tensor, out_host: torch.Tensor,
                            key_mask_host: Optional[torch.Tensor], staging: torch.Tensor, n_groups: int = 0, stream=None) -> None:
    """Forward on host tensors (pinned bf16, dense [tokens, heads, D]) through a device staging buffer; copies of one
    head group overlap the kernels of another.  Synchronise the stream before reading out_host."""
    for t in (q_host, k_host, v_host, out_host):
        if t.is_cuda or t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise ValueError("host tensors must be contiguous CPU bf16 tensors")
    if key_mask_host is not None and (key_mask_host.is_cuda or key_mask_host.dtype != torch.uint8 or not key_mask_host.is_contiguous()):
        raise ValueError("key_mask_host must be a contiguous CPU uint8 tensor")
    if not staging.is_cuda:
        raise ValueError("staging must be a CUDA tensor")
    _check(_lib().sol_attn3d_forward_host(plan, _ptr(q_host), _ptr(k_host), _ptr(v_host), _ptr(out_host), _ptr(key_mask_host),
                                          _ptr(staging), staging.numel() * staging.element_size(), n_groups, _stream(stream)),
           "sol_attn3d_forward_host")


OUT_BF16, OUT_E4M3, OUT_INT8 = 0, 1, 2
MAX_RANKS = 8


def sol_attn3d_forward_e4m3(plan, q, k, v, out_e4m3: torch.Tensor, key_mask=None, stream=None) -> None:
    """Forward whose epilogue writes one raw E4M3 byte per output element (unit scale)."""
    for t in (q, k, v):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v must be CUDA bf16 tensors")
    if not out_e4m3.is_cuda or out_e4m3.element_size() != 1:
        raise ValueError("out_e4m3 must be a CUDA tensor of one-byte elements")
    _check(_lib().sol_attn3d_forward_e4m3(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out_e4m3), _ptr(key_mask),
                                          _stream(stream)), "sol_attn3d_forward_e4m3")


def sol_attn3d_forward_int8(plan, q, k, v, out_records: torch.Tensor, key_mask=None, stream=None) -> None:
    """Forward whose epilogue writes block-INT8 output records [tokens, heads, record_bytes] (uint8)."""
    for t in (q, k, v):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v must be CUDA bf16 tensors")
    if not out_records.is_cuda or out_records.element_size() != 1 or not out_records.is_contiguous():
        raise ValueError("out_records must be a contiguous CUDA tensor of one-byte elements")
    _check(_lib().sol_attn3d_forward_int8(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out_records), _ptr(key_mask),
                                          _stream(stream)), "sol_attn3d_forward_int8")


def sol_attn3d_forward_qkv_int8(plan, qkv_records: torch.Tensor, v_scratch: torch.Tensor, out: torch.Tensor, key_mask=None,
                                out_format: int = OUT_BF16, stream=None) -> None:
    """Forward fed by block-INT8 QKV records [tokens, heads, record_bytes]; v_scratch: bf16 [tokens, heads, D]."""
    if not qkv_records.is_cuda or qkv_records.element_size() != 1 or not qkv_records.is_contiguous():
        raise ValueError("qkv_records must be a contiguous CUDA tensor of one-byte elements")
    if not v_scratch.is_cuda or v_scratch.dtype != torch.bfloat16 or not v_scratch.is_contiguous():
        raise ValueError("v_scratch must be a contiguous CUDA bf16 tensor")
    if not out.is_cuda:
        raise ValueError("out must be a CUDA tensor")
    _check(_lib().sol_attn3d_forward_qkv_int8(plan, _ptr(qkv_records), _ptr(v_scratch), _ptr(out), _ptr(key_mask), out_format,
                                              _stream(stream)), "sol_attn3d_forward_qkv_int8")


def _ptr_array(ptrs: Sequence[int]):
    return (ctypes.c_void_p * len(ptrs))(*[ctypes.c_void_p(int(x)) if x else None for x in ptrs])


def sol_attn3d_forward_scatter(plan, q, k, v, key_mask, dst: Sequence[int], tok_begin: Sequence[int], dst_heads: int,
                               head_offset: int, out_format: int = OUT_BF16, stream=None) -> None:
    """dst: device addresses (ints; this GPU's or peer-mapped) of the token owners' [n_g, dst_heads, D] buffers."""
    for t in (q, k, v):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v must be CUDA bf16 tensors")
    if len(tok_begin) != len(dst) + 1:
        raise ValueError("tok_begin needs len(dst) + 1 entries")
    tb = (ctypes.c_int64 * len(tok_begin))(*[int(x) for x in tok_begin])
    _check(_lib().sol_attn3d_forward_scatter(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(key_mask), len(dst), _ptr_array(dst),
                                             tb, dst_heads, head_offset, out_format, _stream(stream)),
           "sol_attn3d_forward_scatter")


_I64x2, _I64x3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3


def _strides_of(t: torch.Tensor, head_dim: int):
    """(token, head) element strides of a [tokens, heads, head_dim] tensor whose head_dim axis is contiguous."""
    shape, st = t.shape, t.stride()
    if len(shape) != 3 or shape[2] != head_dim or st[2] != 1:
        raise ValueError("expected [tokens, heads, head_dim] with contiguous head_dim")
    # the stride torch reports for an axis of extent 0 or 1 is arbitrary: use the dense value there
    return _I64x2(st[0] if shape[0] > 1 else shape[1] * head_dim, st[1] if shape[1] > 1 else head_dim)


def sol_attn3d_exchange_pack_qkv(q, k, v, n_ranks: int, dst: Sequence[int], dst_row0: int = 0, stream=None,
                                 group_begin: int = 0, group_heads: int = 0) -> None:
    """q, k, v: CUDA bf16 [n_local, heads, D] (any token / head strides); dst: n_ranks device addresses.
    group_begin / group_heads: send only that head group of every rank's shard (0, 0 = the whole shard)."""
    n_local, heads, head_dim = q.shape
    for t in (q, k, v):
        if not t.is_cuda or t.dtype != torch.bfloat16 or tuple(t.shape) != (n_local, heads, head_dim):
            raise ValueError("q, k, v must be CUDA bf16 tensors of one shape")
    if len(dst) != n_ranks:
        raise ValueError("one destination per rank")
    _check(_lib().sol_attn3d_exchange_pack_qkv(_ptr(q), _ptr(k), _ptr(v), _strides_of(q, head_dim), _strides_of(k, head_dim),
                                               _strides_of(v, head_dim), n_local, heads, head_dim, n_ranks, group_begin,
                                               group_heads, _ptr_array(dst), dst_row0, _stream(stream)),
           "sol_attn3d_exchange_pack_qkv")


WIRE_QKV_BF16, WIRE_QKV_INT8, WIRE_OUT_BF16, WIRE_OUT_E4M3, WIRE_OUT_INT8 = 0, 1, 2, 3, 4


def sol_attn3d_exchange_record_bytes(kind: int, head_dim: int) -> int:
    n = int(_lib().sol_attn3d_exchange_record_bytes(kind, head_dim))
    if n == 0:
        raise ValueError("unknown wire format or head_dim")
    return n


def sol_attn3d_exchange_pack_qkv_int8(q, k, v, n_ranks: int, dst: Sequence[int], dst_row0: int = 0, stream=None,
                                      group_begin: int = 0, group_heads: int = 0) -> None:
    """As sol_attn3d_exchange_pack_qkv, but the destinations receive block-INT8 records."""
    n_local, heads, head_dim = q.shape
    for t in (q, k, v):
        if not t.is_cuda or t.dtype != torch.bfloat16 or tuple(t.shape) != (n_local, heads, head_dim):
            raise ValueError("q, k, v must be CUDA bf16 tensors of one shape")
    if len(dst) != n_ranks:
        raise ValueError("one destination per rank")
    _check(_lib().sol_attn3d_exchange_pack_qkv_int8(_ptr(q), _ptr(k), _ptr(v), _strides_of(q, head_dim),
                                                    _strides_of(k, head_dim), _strides_of(v, head_dim), n_local, heads,
                                                    head_dim, n_ranks, group_begin, group_heads, _ptr_array(dst), dst_row0,
                                                    _stream(stream)),
           "sol_attn3d_exchange_pack_qkv_int8")


def sol_attn3d_exchange_unpack_qkv_int8(records: torch.Tensor, qkv: torch.Tensor, n_rows: int, heads: int, head_dim: int,
                                        stream=None) -> None:
    if not records.is_cuda or not qkv.is_cuda or qkv.dtype != torch.bfloat16 or not qkv.is_contiguous():
        raise ValueError("records: CUDA bytes; qkv: contiguous CUDA bf16 [rows, 3, heads, D]")
    _check(_lib().sol_attn3d_exchange_unpack_qkv_int8(_ptr(records), _ptr(qkv), n_rows, heads, head_dim, _stream(stream)),
           "sol_attn3d_exchange_unpack_qkv_int8")


def sol_attn3d_exchange_quantize_out_int8(out_rows: torch.Tensor, records: torch.Tensor, stream=None) -> None:
    n_rows, heads, head_dim = out_rows.shape
    if not out_rows.is_cuda or out_rows.dtype != torch.bfloat16 or not records.is_cuda:
        raise ValueError("out_rows: CUDA bf16 [rows, heads, D]; records: CUDA bytes")
    _check(_lib().sol_attn3d_exchange_quantize_out_int8(_ptr(out_rows), _strides_of(out_rows, head_dim), n_rows, heads,
                                                        head_dim, _ptr(records), _stream(stream)),
           "sol_attn3d_exchange_quantize_out_int8")


def sol_attn3d_exchange_dequantize_out_int8(records: torch.Tensor, out_rows: torch.Tensor, stream=None) -> None:
    n_rows, heads, head_dim = out_rows.shape
    if not out_rows.is_cuda or out_rows.dtype != torch.bfloat16 or not out_rows.is_contiguous() or not records.is_cuda:
        raise ValueError("out_rows: contiguous CUDA bf16 [rows, heads, D]; records: CUDA bytes")
    _check(_lib().sol_attn3d_exchange_dequantize_out_int8(_ptr(records), _ptr(out_rows), n_rows, heads, head_dim,
                                                          _stream(stream)), "sol_attn3d_exchange_dequantize_out_int8")


def sol_attn3d_exchange_merge_heads(recv: torch.Tensor, out, n_local: int, heads: int, record_bytes: int,
                                    n_ranks: int, out_tok_stride_bytes: int = 0, stream=None, out_rank_stride_bytes: int = 0) -> None:
    """out: CUDA tensor, or a device address (int) when the rows start inside a larger tensor."""
    if not recv.is_cuda or not recv.is_contiguous():
        raise ValueError("recv must be a contiguous CUDA tensor")
    out_ptr = ctypes.c_void_p(int(out)) if isinstance(out, int) else _ptr(out)
    _check(_lib().sol_attn3d_exchange_merge_heads(_ptr(recv), out_ptr, n_local, heads, record_bytes, n_ranks,
                                                  out_tok_stride_bytes, out_rank_stride_bytes, _stream(stream)),
           "sol_attn3d_exchange_merge_heads")


def sol_attn3d_sparse_workspace_bytes(plan) -> int:
    return int(_lib().sol_attn3d_sparse_workspace_bytes(plan))


def sol_attn3d_forward_sparse(plan, q, k, v, out, key_mask, tau: float, sparse_ws: torch.Tensor, stream=None) -> None:
    """Block-sparse forward (mu + tau*sigma selection of 128-key blocks per 256-row query block)."""
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    _check(_lib().sol_attn3d_forward_sparse(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask),
                                            ctypes.c_float(tau), _ptr(sparse_ws),
                                            sparse_ws.numel() * sparse_ws.element_size(), _stream(stream)),
           "sol_attn3d_forward_sparse")


def sol_attn3d_sparse_stats(plan, sparse_ws: torch.Tensor) -> Tuple[int, int]:
    a, b = ctypes.c_longlong(), ctypes.c_longlong()
    _check(_lib().sol_attn3d_sparse_stats(plan, _ptr(sparse_ws), ctypes.byref(a), ctypes.byref(b)), "sol_attn3d_sparse_stats")
    return int(a.value), int(b.value)


def sol_attn3d_sparse_selection(plan, sparse_ws: torch.Tensor, seq: int, head: int, query_block: int, capacity: int) -> list:
    buf = (ctypes.c_int * max(capacity, 1))()
    n = ctypes.c_int()
    _check(_lib().sol_attn3d_sparse_selection(plan, _ptr(sparse_ws), seq, head, query_block, buf, capacity,
                                              ctypes.byref(n)), "sol_attn3d_sparse_selection")
    return [int(buf[i]) for i in range(min(n.value, capacity))]


def _check_gain(g: torch.Tensor, head_dim_hint=None):
    if g is None or not g.is_cuda or g.dtype != torch.float32 or not g.is_contiguous():
        raise ValueError("gains must be contiguous CUDA float32 tensors of head_dim elements")


def sol_attn3d_forward_qknorm(plan, q, k, v, out, key_mask, q_gain: torch.Tensor, k_gain: torch.Tensor, eps: float,
                              stream=None) -> None:
    """Forward with QK RMS-norm (gain vectors of head_dim fp32 values) applied before the rotary embedding."""
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    _check_gain(q_gain)
    _check_gain(k_gain)
    _check(_lib().sol_attn3d_forward_qknorm(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask), _ptr(q_gain),
                                            _ptr(k_gain), ctypes.c_float(eps), _stream(stream)),
           "sol_attn3d_forward_qknorm")


def sol_attn3d_qknorm_rope(plan, q, k, q_gain, k_gain, eps: float, q_out, k_out, stream=None) -> None:
    _check(_lib().sol_attn3d_qknorm_rope(plan, _ptr(q), _ptr(k), _ptr(q_gain), _ptr(k_gain), ctypes.c_float(eps),
                                         _ptr(q_out), _ptr(k_out), _stream(stream)), "sol_attn3d_qknorm_rope")


class sol_attn3d_diff_weights:
    """Learned weights of the differential attention: keeps the tensors alive and marshals them.

    lambda_*: contiguous CUDA fp32, [64] (shared by the head pairs) or [pairs, 64]; gain: [128] or None (no norm)."""

    def __init__(self, lambda_q1, lambda_k1, lambda_q2, lambda_k2, lambda_init: float, gain: Optional[torch.Tensor] = None,
                 eps: float = 1e-5):
        vecs = (lambda_q1, lambda_k1, lambda_q2, lambda_k2)
        for t in vecs:
            if not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or t.shape != lambda_q1.shape or \
                    t.dim() not in (1, 2) or t.shape[-1] != 64:
                raise ValueError("lambda vectors must be contiguous CUDA float32 tensors of one shape, [64] or [pairs, 64]")
        if gain is not None and (not gain.is_cuda or gain.dtype != torch.float32 or not gain.is_contiguous() or gain.numel() != 128):
            raise ValueError("gain must be a contiguous CUDA float32 tensor of 128 elements")
        self.tensors = vecs + (gain,)
        self.pairs = lambda_q1.shape[0] if lambda_q1.dim() == 2 else None
        self.struct = _DiffWeights(ctypes.sizeof(_DiffWeights), lambda_init, *(t.data_ptr() for t in vecs),
                                   64 if self.pairs is not None else 0, None if gain is None else gain.data_ptr(), eps)


def _check_pairs(weights: sol_attn3d_diff_weights, heads: int) -> None:
    if weights.pairs is not None and weights.pairs != heads // 2:
        raise ValueError("one set of lambda vectors, or one per head pair")


def sol_attn3d_forward_diff(plan, q, k, v, out, key_mask, weights: sol_attn3d_diff_weights,
                            query_mask: Optional[torch.Tensor] = None, stream=None) -> None:
    """Differential attention over a plan with head_dim 64: heads 2i, 2i+1 are two softmax maps over one 128-dim value."""
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    for m, name in ((key_mask, "key_mask"), (query_mask, "query_mask")):
        if m is not None and (not m.is_cuda or m.dtype != torch.uint8 or not m.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous CUDA uint8 tensor")
    _, heads, head_dim, tokens = sol_attn3d_plan_dims(plan)
    _check_sizes(tokens, heads * head_dim, (q, k, v, out), (key_mask, query_mask))
    _check_pairs(weights, heads)
    _check_on_device(q, k, v, out, key_mask, query_mask, *weights.tensors)
    _check(_lib().sol_attn3d_forward_diff(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask), _ptr(query_mask),
                                          ctypes.byref(weights.struct), _stream(stream)), "sol_attn3d_forward_diff")


def _check_sizes(tokens: int, row: int, tensors, masks) -> None:
    """The kernels go by the plan, whatever the tensors' shapes say: refuse what is too small for it."""
    for t in tensors:
        if t.numel() < tokens * row:
            raise ValueError(f"q, k, v, out: the plan has {tokens} tokens of {row} values")
    for m in masks:
        if m is not None and m.numel() < tokens:
            raise ValueError(f"masks: the plan has {tokens} tokens")


def _check_on_device(*tensors) -> None:
    """The library launches on the current device: refuse tensors that live on another one."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"tensor on {t.device}, current device is cuda:{here}")


def _check_index(t: Optional[torch.Tensor], n: int, name: str) -> None:
    if t is not None and (not t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous() or t.numel() != n):
        raise ValueError(f"{name} must be a contiguous CUDA int32 tensor with one element per row")


def sol_attn3d_diff_step_workspace_bytes(batch: int, heads: int, head_dim: int, capacity: int) -> int:
    return int(_lib().sol_attn3d_diff_step_workspace_bytes(batch, heads, head_dim, capacity))


_DENSE2, _DENSE3 = _I64x2(0, 0), _I64x3(0, 0, 0)         # strides of a contiguous tensor, for calls that take 0 as "dense"


def _row_strides(t: torch.Tensor, head_dim: int):
    """_strides_of for calls that take 0 as "dense": an expanded axis is refused."""
    st = _strides_of(t, head_dim)
    if st[0] == 0 or st[1] == 0:
        raise ValueError("expanded tensors (stride 0) are not supported")
    return st


def _cache_strides(t: torch.Tensor, shape):
    st = t.stride()
    if t.shape != shape or st[3] != 1:
        raise ValueError("caches: [slots, capacity, heads, head_dim] of one shape with contiguous head_dim")
    if 0 in st and any(s == 0 and n > 1 for s, n in zip(st, shape)):
        raise ValueError("expanded tensors (stride 0) are not supported")
    # the stride torch reports for an axis of extent 0 or 1 is arbitrary: 0 asks for the dense value there
    return _I64x3(st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0, st[2] if shape[2] > 1 else 0)


def sol_attn3d_diff_step(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, lens: torch.Tensor, out: torch.Tensor,
                         weights: sol_attn3d_diff_weights, workspace: Optional[torch.Tensor],
                         key_mask: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, stream=None) -> None:
    """One query token per row, q, out [batch, heads, 64], over caches [slots, capacity, heads, 64] (all rotated)."""
    batch, heads, head_dim = q.shape
    for t in (q, k_cache, v_cache, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, caches and out must be CUDA bf16 tensors")
    shape = k_cache.shape
    if out.shape != q.shape or len(shape) != 4 or shape[2:] != q.shape[1:] or v_cache.shape != shape:
        raise ValueError("q, out: [batch, heads, 64]; caches: [slots, capacity, heads, 64]")
    _check_index(lens, batch, "lens")
    _check_index(slots, batch, "slots")
    if key_mask is not None and (not key_mask.is_cuda or key_mask.dtype != torch.uint8 or not key_mask.is_contiguous() or
                                 key_mask.shape != shape[:2]):
        raise ValueError("key_mask must be a contiguous CUDA uint8 tensor [slots, capacity]")
    _check_pairs(weights, heads)
    _check_on_device(q, k_cache, v_cache, lens, out, workspace, key_mask, slots, *weights.tensors)
    cache = _KvCache(_KV_CACHE_SIZE, k_cache.data_ptr(), v_cache.data_ptr(),
                     _DENSE3 if k_cache.is_contiguous() else _cache_strides(k_cache, shape),
                     _DENSE3 if v_cache.is_contiguous() else _cache_strides(v_cache, shape), shape[0], shape[1], _ptr(key_mask), 0)
    nbytes = 0 if workspace is None else workspace.nbytes
    _check(_lib().sol_attn3d_diff_step(_ptr(q), _DENSE2 if q.is_contiguous() else _row_strides(q, head_dim), ctypes.byref(cache), _ptr(lens), _ptr(slots), _ptr(out),
                                       _DENSE2 if out.is_contiguous() else _row_strides(out, head_dim), batch, heads, head_dim,
                                       ctypes.byref(weights.struct), _ptr(workspace), nbytes, _stream(stream)), "sol_attn3d_diff_step")


def sol_attn3d_linear_workspace_bytes(plan) -> int:
    return int(_lib().sol_attn3d_linear_workspace_bytes(plan))


def sol_attn3d_forward_linear(plan, q, k, v, out, key_mask, log_decay: torch.Tensor, scale: float,
                              state_in: Optional[torch.Tensor] = None, state_out: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Causal linear attention with a decay per head over a plan; states fp32 [sequences, heads, D, D]."""
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors")
    if key_mask is not None and (not key_mask.is_cuda or key_mask.dtype != torch.uint8 or not key_mask.is_contiguous()):
        raise ValueError("key_mask must be a contiguous CUDA uint8 tensor")
    n_seqs, heads, head_dim, tokens = sol_attn3d_plan_dims(plan)
    _check_sizes(tokens, heads * head_dim, (q, k, v, out), (key_mask,))
    for t in (state_in, state_out):
        if t is not None and (not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or
                              t.shape != (n_seqs, heads, head_dim, head_dim)):
            raise ValueError(f"states must be contiguous CUDA float32 tensors, {[n_seqs, heads, head_dim, head_dim]} for this plan")
    _check_decay(log_decay, heads)
    _check_on_device(q, k, v, out, key_mask, log_decay, state_in, state_out, workspace)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib().sol_attn3d_forward_linear(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(key_mask), _ptr(log_decay),
                                            ctypes.c_float(scale), _ptr(state_in), _ptr(state_out), _ptr(workspace), nbytes,
                                            _stream(stream)), "sol_attn3d_forward_linear")


def sol_attn3d_linear_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, log_decay: torch.Tensor,
                           scale: float, state_in: torch.Tensor, state_out: torch.Tensor, slots: Optional[torch.Tensor] = None,
                           stream=None) -> None:
    """One token per row, q, k, v, out [batch, heads, D]; states fp32 [slots, heads, D, D], in place or not."""
    batch, heads, head_dim = q.shape
    for t in (q, k, v, out):
        if not t.is_cuda or t.dtype != torch.bfloat16 or t.shape != q.shape:
            raise ValueError("q, k, v, out must be CUDA bf16 tensors of one shape")
    want = (state_in.shape[0], heads, head_dim, head_dim)
    for t in (state_in, state_out):
        if not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous() or t.shape != want:
            raise ValueError("states must be contiguous CUDA float32 tensors [slots, heads, D, D]")
    _check_decay(log_decay, heads)
    _check_index(slots, batch, "slots")
    _check_on_device(q, k, v, out, log_decay, state_in, state_out, slots)
    st = [_DENSE2 if t.is_contiguous() else _row_strides(t, head_dim) for t in (q, k, v, out)]
    _check(_lib().sol_attn3d_linear_step(_ptr(q), _ptr(k), _ptr(v), _ptr(out), *st, batch, heads, head_dim, _ptr(log_decay), scale,
                                         _ptr(state_in), _ptr(state_out), want[0], _ptr(slots), _stream(stream)),
           "sol_attn3d_linear_step")


def _check_decay(log_decay: torch.Tensor, heads: int) -> None:
    if not log_decay.is_cuda or log_decay.dtype != torch.float32 or not log_decay.is_contiguous() or log_decay.numel() != heads:
        raise ValueError("log_decay must be a contiguous CUDA float32 tensor with one element per head")


def _dims(plan) -> Tuple[int, int, int, int]:
    """sol_attn3d_plan_dims, asked once per handle."""
    dims = getattr(plan, "dims", None)
    if dims is None:
        dims = sol_attn3d_plan_dims(plan)
        if isinstance(plan, _Plan):
            plan.dims = dims
    return dims


_shared_strides = functools.lru_cache(maxsize=1024)(_I64x2)      # arrays that are only read


def _shared_row_strides(t: torch.Tensor, head_dim: int):
    """_row_strides without building an array for every call."""
    if t.is_contiguous():
        return _DENSE2
    shape, st = t.shape, t.stride()
    if shape[2] != head_dim or st[2] != 1:
        raise ValueError("expected [tokens, heads, head_dim] with contiguous head_dim")
    s0, s1 = st[0] if shape[0] > 1 else shape[1] * head_dim, st[1] if shape[1] > 1 else head_dim
    if s0 == 0 or s1 == 0:
        raise ValueError("expanded tensors (stride 0) are not supported")
    return _shared_strides(s0, s1)


def _one_device(tensors) -> int:
    """The device that all of them live on."""
    device = tensors[0].get_device()
    if any(t.get_device() != device for t in tensors):
        raise ValueError("all tensors must be on one device")
    return device


def _check_here(device: int, *tensors) -> None:
    """_check_on_device for a holder of tensors (all on `device`) and some more."""
    here = torch._C._cuda_getDevice()
    if device != here:
        raise ValueError(f"tensors on cuda:{device}, current device is cuda:{here}")
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"tensor on {t.device}, current device is cuda:{here}")


_NO_STRIDES = dict.fromkeys(("q", "out"))


def _check_strides(plan, name: str, t: torch.Tensor, heads: int, head_dim: int) -> None:
    """The kernels take q and out by the plan's strides.  A tensor of the shape [tokens, heads, head_dim], or [tokens, heads * head_dim], has to
    have them; any other is memory that the plan's strides lead through."""
    want, st = getattr(plan, "strides", None), t.stride()
    if want is None or st == want[name]:
        return
    (tok, head, _), shape = want[name], t.shape
    if len(shape) == 3 and shape[1] == heads and shape[2] == head_dim:
        same = st[2] == 1 and (heads == 1 or st[1] == head)
    elif len(shape) == 2 and shape[1] == heads * head_dim:
        same = st[1] == 1 and (heads == 1 or head == head_dim)
    else:
        return
    if not same or (shape[0] > 1 and st[0] != tok):
        raise ValueError(f"{name}: strides {st}, but the plan was made for {want[name]}")


def _check_plan(plan, here: int) -> None:
    if getattr(plan, "device", here) != here:
        raise ValueError(f"the plan's workspace is on cuda:{plan.device}, current device is cuda:{here}")


def _pool_strides(t: torch.Tensor, extents, n: int):
    """Element strides of all axes but the last; 0 (the dense value) where torch's is arbitrary (extent 0 or 1)."""
    st = t.stride()
    if st[-1] != 1 and extents[-1] > 1:
        raise ValueError("head_dim must be contiguous")
    if any(s == 0 and e > 1 for s, e in zip(st, extents)):
        raise ValueError("expanded tensors (stride 0) are not supported")
    return (ctypes.c_int64 * n)(*(s if e > 1 else 0 for s, e in zip(st[:-1], extents)))


class sol_attn3d_paged_cache:
    """A K/V cache in pages: keeps the tensors alive and marshals them.

    k, v: CUDA bf16 [layers, pages, page_size, kv_heads, head_dim]; table: int32 [streams, columns], lens: int32 [streams],
    refs: int32 [pages] (streams that hold a page), or None for a cache that is only read and appended to."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, refs: Optional[torch.Tensor] = None):
        for t in (k, v):
            if not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != 5 or t.shape != k.shape:
                raise ValueError("k, v must be CUDA bf16 tensors [layers, pages, page_size, kv_heads, head_dim] of one shape")
        for t, dims, name in ((table, 2, "table"), (lens, 1, "lens"), (refs, 1, "refs")):
            if t is not None and (not t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous() or t.dim() != dims):
                raise ValueError(f"{name} must be a contiguous CUDA int32 tensor of {dims} dimension(s)")
        if lens.shape[0] != table.shape[0] or (refs is not None and refs.shape[0] != k.shape[1]):
            raise ValueError("lens has one element per row of the table, refs one per page")
        layers, pages, page, kv_heads, head_dim = k.shape
        self.k, self.v, self.table, self.lens, self.refs = k, v, table, lens, refs
        self.tensors = (k, v, table, lens) + (() if refs is None else (refs,))
        self.device = _one_device(self.tensors)
        self.kv_heads, self.head_dim, self.n_streams = kv_heads, head_dim, table.shape[0]
        self.struct = _PagedCache(ctypes.sizeof(_PagedCache), layers, page, kv_heads, head_dim, k.data_ptr(), v.data_ptr(),
                                  _pool_strides(k, k.shape, 4), _pool_strides(v, v.shape, 4), pages, table.data_ptr(), lens.data_ptr(),
                                  _ptr(refs), table.shape[0], table.shape[1])
        self.ref = ctypes.byref(self.struct)


class sol_attn3d_context:
    """Encoder states to attend to: keeps the tensors alive and marshals them.

    k, v: CUDA bf16 [rows, kv_heads, head_dim]; begins, lens: int32, one per sequence (or row, for the step form); no length is
    larger than max_len; key_mask: uint8 [rows] or None."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, begins: torch.Tensor, lens: torch.Tensor, max_len: int,
                 key_mask: Optional[torch.Tensor] = None):
        for t in (k, v):
            if not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != 3 or t.shape != k.shape:
                raise ValueError("k, v must be CUDA bf16 tensors [rows, kv_heads, head_dim] of one shape")
        _check_index(begins, begins.numel(), "begins")
        _check_index(lens, begins.numel(), "lens")
        if key_mask is not None and (not key_mask.is_cuda or key_mask.dtype != torch.uint8 or not key_mask.is_contiguous() or
                                     key_mask.numel() != k.shape[0]):
            raise ValueError("key_mask must be a contiguous CUDA uint8 tensor with one element per row")
        self.tensors = (k, v, begins, lens) + (() if key_mask is None else (key_mask,))
        self.device = _one_device(self.tensors)
        self.k, self.v, self.begins, self.lens, self.key_mask = k, v, begins, lens, key_mask
        self.kv_heads, self.head_dim, self.n = k.shape[1], k.shape[2], begins.numel()
        self.struct = _Context(ctypes.sizeof(_Context), k.shape[1], k.shape[2], k.data_ptr(), v.data_ptr(), _pool_strides(k, k.shape, 2),
                               _pool_strides(v, v.shape, 2), k.shape[0], begins.data_ptr(), lens.data_ptr(), max_len, _ptr(key_mask))
        self.ref = ctypes.byref(self.struct)


def _check_workspace(t: Optional[torch.Tensor]) -> int:
    if t is None:
        return 0
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor")
    return t.nbytes


def _check_requests(cache: sol_attn3d_paged_cache, status, *lists) -> int:
    n = lists[0].numel()
    if cache.refs is None:
        raise ValueError("this cache keeps no count of the streams that hold a page (refs)")
    here = torch._C._cuda_getDevice()
    if cache.device != here:
        raise ValueError(f"the cache is on cuda:{cache.device}, current device is cuda:{here}")
    for t in lists if status is None else (status,) + lists:
        if t.dtype is not torch.int32 or t.get_device() != here or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"streams, parents, amounts, status must be contiguous int32 tensors of one size on cuda:{here}")
    return n


def sol_attn3d_cache_workspace_bytes(cache: sol_attn3d_paged_cache, n: int) -> int:
    return int(_lib().sol_attn3d_cache_workspace_bytes(cache.ref, n))


def sol_attn3d_cache_reserve(cache: sol_attn3d_paged_cache, streams: torch.Tensor, amount: torch.Tensor,
                             status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Stream streams[i] grows by amount[i] tokens and the pages that they need; status[i] says whether it did (CACHE_*)."""
    n = _check_requests(cache, status, streams, amount)
    _check(_lib().sol_attn3d_cache_reserve(cache.ref, n, _ptr(streams), _ptr(amount), _ptr(status), _stream(stream)), "sol_attn3d_cache_reserve")


def sol_attn3d_cache_fork(cache: sol_attn3d_paged_cache, parents: torch.Tensor, streams: torch.Tensor, status: Optional[torch.Tensor],
                          workspace: torch.Tensor, stream=None) -> None:
    """The empty stream streams[i] becomes a branch of parents[i]."""
    n = _check_requests(cache, status, parents, streams)
    nbytes = _check_workspace(workspace)
    _check_on_device(workspace)
    _check(_lib().sol_attn3d_cache_fork(cache.ref, n, _ptr(parents), _ptr(streams), _ptr(status), _ptr(workspace), nbytes, _stream(stream)),
           "sol_attn3d_cache_fork")


def sol_attn3d_cache_compact(cache: sol_attn3d_paged_cache, streams: torch.Tensor, keep: torch.Tensor, status: Optional[torch.Tensor],
                             workspace: torch.Tensor, stream=None) -> None:
    """Of stream streams[i] the tokens with keep[i] != 0 stay; keep: uint8 [len(streams), width], tokens beyond the width go."""
    n = _check_requests(cache, status, streams)
    if not keep.is_cuda or keep.dtype != torch.uint8 or not keep.is_contiguous() or keep.dim() != 2 or keep.shape[0] != n:
        raise ValueError("keep must be a contiguous CUDA uint8 tensor with one row per stream")
    nbytes = _check_workspace(workspace)
    _check_on_device(keep, workspace)
    _check(_lib().sol_attn3d_cache_compact(cache.ref, n, _ptr(streams), _ptr(keep), keep.shape[1], _ptr(status), _ptr(workspace), nbytes,
                                           _stream(stream)), "sol_attn3d_cache_compact")


def sol_attn3d_cache_free(cache: sol_attn3d_paged_cache, streams: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """The streams give their pages back and are empty."""
    n = _check_requests(cache, status, streams)
    _check(_lib().sol_attn3d_cache_free(cache.ref, n, _ptr(streams), _ptr(status), _stream(stream)), "sol_attn3d_cache_free")


def sol_attn3d_cache_copy_pages(cache: sol_attn3d_paged_cache, src_pages: torch.Tensor, dst_pages: torch.Tensor, stream=None) -> None:
    """Page dst_pages[i] = page src_pages[i], in all layers."""
    n = src_pages.numel()
    _check_index(src_pages, n, "src_pages")
    _check_index(dst_pages, n, "dst_pages")
    _check_here(cache.device, src_pages, dst_pages)
    _check(_lib().sol_attn3d_cache_copy_pages(cache.ref, n, _ptr(src_pages), _ptr(dst_pages), _stream(stream)), "sol_attn3d_cache_copy_pages")


def _check_bf16(*tensors) -> None:
    for t in tensors:
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("tensors must be CUDA bf16 tensors")


def sol_attn3d_cache_append(plan, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, q_out: Optional[torch.Tensor],
                            cache: sol_attn3d_paged_cache, layer: int, streams: Optional[torch.Tensor] = None,
                            pos0: Optional[torch.Tensor] = None, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None,
                            eps: float = 0.0, stream=None) -> None:
    """Norm and rotation of new tokens; K and V go to the last tokens of their streams, Q to q_out."""
    n_seqs, heads, head_dim, tokens = getattr(plan, "dims", None) or _dims(plan)
    here = torch._C._cuda_getDevice()
    if cache.device != here:
        raise ValueError(f"the cache is on cuda:{cache.device}, current device is cuda:{here}")
    if getattr(plan, "device", here) != here:
        _check_plan(plan, here)
    # (a tensor on the CPU has device -1)
    for t in (k, v, q, q_out):
        if t is not None and (t.dtype is not torch.bfloat16 or t.get_device() != here):
            raise ValueError(f"q, k, v, q_out must be bf16 tensors on cuda:{here}")
    for t in (q, q_out):
        if t is not None and t.numel() < tokens * heads * head_dim:
            raise ValueError(f"q, q_out: the plan has {tokens} tokens of {heads * head_dim} values")
    if q is not None and q.stride() != getattr(plan, "strides", _NO_STRIDES)["q"]:
        _check_strides(plan, "q", q, heads, head_dim)
    if q_out is not None and not q_out.is_contiguous():
        raise ValueError("q_out must be contiguous")
    want = (tokens, cache.kv_heads, cache.head_dim)
    if k.shape != want or v.shape != want:
        raise ValueError(f"k, v: {list(want)} for this plan and cache")
    for t, n, name in ((streams, n_seqs, "streams"), (pos0, 3 * n_seqs, "pos0")):
        if t is not None and (t.dtype is not torch.int32 or t.get_device() != here or t.numel() != n or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous int32 tensor of {n} elements on cuda:{here}")
    for g in (q_gain, k_gain):
        if g is not None and (g.dtype is not torch.float32 or g.get_device() != here or g.numel() != head_dim or not g.is_contiguous()):
            raise ValueError(f"gains must be contiguous float32 tensors of {head_dim} elements on cuda:{here}")
    ks = _shared_row_strides(k, head_dim)    # (K and V are mostly slices of one tensor)
    vs = ks if ks is not _DENSE2 and v.stride() == k.stride() else _shared_row_strides(v, head_dim)
    code = _lib().sol_attn3d_cache_append(
        plan, None if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(), ks, vs,
        None if q_out is None else q_out.data_ptr(), cache.ref, layer, None if streams is None else streams.data_ptr(),
        None if pos0 is None else pos0.data_ptr(), None if q_gain is None else q_gain.data_ptr(),
        None if k_gain is None else k_gain.data_ptr(), eps, _stream(stream))
    if code != OK:
        raise SolAttn3dError(code, "sol_attn3d_cache_append")


def _check_key_mask(cache: sol_attn3d_paged_cache, key_mask: Optional[torch.Tensor]) -> int:
    if key_mask is None:
        return 0
    if not key_mask.is_cuda or key_mask.dtype != torch.uint8 or not key_mask.is_contiguous() or key_mask.dim() != 2 or \
            key_mask.shape[0] != cache.n_streams:
        raise ValueError("key_mask must be a contiguous CUDA uint8 tensor [streams, tokens]")
    if key_mask.shape[1] == 0:               # (its address is null, which would mean "no mask")
        raise ValueError("key_mask has no columns")
    return key_mask.shape[1]


def sol_attn3d_paged_workspace_bytes(plan, cache: sol_attn3d_paged_cache) -> int:
    return int(_lib().sol_attn3d_paged_workspace_bytes(plan, cache.ref))


def sol_attn3d_forward_paged(plan, q: torch.Tensor, cache: sol_attn3d_paged_cache, layer: int, out: torch.Tensor,
                             streams: Optional[torch.Tensor] = None, key_mask: Optional[torch.Tensor] = None, causal_block: int = 0,
                             workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """The plan's sequences are the last tokens of streams of the cache and attend to them; causal_block: see the header."""
    n_seqs, heads, head_dim, tokens = _dims(plan)
    _check_bf16(q, out)
    _check_sizes(tokens, heads * head_dim, (q, out), ())
    _check_strides(plan, "q", q, heads, head_dim)
    _check_strides(plan, "out", out, heads, head_dim)
    _check_index(streams, n_seqs, "streams")
    width = _check_key_mask(cache, key_mask)
    nbytes = _check_workspace(workspace)
    _check_here(cache.device, q, out, streams, key_mask, workspace)
    _check_plan(plan, cache.device)
    _check(_lib().sol_attn3d_forward_paged(plan, _ptr(q), cache.ref, layer, _ptr(out), _ptr(streams), _ptr(key_mask), width, causal_block,
                                           _ptr(workspace), nbytes, _stream(stream)), "sol_attn3d_forward_paged")


def sol_attn3d_paged_step_workspace_bytes(cache: sol_attn3d_paged_cache, batch: int, heads: int) -> int:
    return int(_lib().sol_attn3d_paged_step_workspace_bytes(cache.ref, batch, heads))


def _check_rows(q: torch.Tensor, out: torch.Tensor, head_dim: int) -> None:
    _check_bf16(q, out)
    if q.dim() != 3 or q.shape != out.shape or q.shape[2] != head_dim:
        raise ValueError(f"q, out: [batch, heads, {head_dim}]")


def sol_attn3d_paged_step(q: torch.Tensor, cache: sol_attn3d_paged_cache, layer: int, out: torch.Tensor,
                          streams: Optional[torch.Tensor] = None, key_mask: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """One token per row, q, out [batch, heads, D]: the last token of its stream, over all of the stream."""
    head_dim = cache.head_dim
    _check_rows(q, out, head_dim)
    batch, heads = q.shape[0], q.shape[1]
    _check_index(streams, batch, "streams")
    width = _check_key_mask(cache, key_mask)
    nbytes = _check_workspace(workspace)
    _check_here(cache.device, q, out, streams, key_mask, workspace)
    _check(_lib().sol_attn3d_paged_step(_ptr(q), _shared_row_strides(q, head_dim), cache.ref, layer, _ptr(streams),
                                        _ptr(out), _shared_row_strides(out, head_dim), batch, heads,
                                        _ptr(key_mask), width, _ptr(workspace), nbytes, _stream(stream)), "sol_attn3d_paged_step")


def sol_attn3d_cross_workspace_bytes(plan, context: sol_attn3d_context) -> int:
    return int(_lib().sol_attn3d_cross_workspace_bytes(plan, context.ref))


def sol_attn3d_forward_cross(plan, q: torch.Tensor, context: sol_attn3d_context, out: torch.Tensor,
                             workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Cross attention of the plan's sequences, each to its context."""
    n_seqs, heads, head_dim, tokens = _dims(plan)
    _check_bf16(q, out)
    _check_sizes(tokens, heads * head_dim, (q, out), ())
    _check_strides(plan, "q", q, heads, head_dim)
    _check_strides(plan, "out", out, heads, head_dim)
    if context.n != n_seqs:
        raise ValueError(f"{n_seqs} sequences need as many contexts")
    nbytes = _check_workspace(workspace)
    _check_here(context.device, q, out, workspace)
    _check_plan(plan, context.device)
    _check(_lib().sol_attn3d_forward_cross(plan, _ptr(q), context.ref, _ptr(out), _ptr(workspace), nbytes, _stream(stream)),
           "sol_attn3d_forward_cross")


def sol_attn3d_cross_step_workspace_bytes(context: sol_attn3d_context, batch: int, heads: int) -> int:
    return int(_lib().sol_attn3d_cross_step_workspace_bytes(context.ref, batch, heads))


def sol_attn3d_cross_step(q: torch.Tensor, context: sol_attn3d_context, out: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    """One row per context, q, out [batch, heads, D]."""
    head_dim = context.head_dim
    _check_rows(q, out, head_dim)
    batch, heads = q.shape[0], q.shape[1]
    if context.n != batch:
        raise ValueError("one context per row")
    nbytes = _check_workspace(workspace)
    _check_here(context.device, q, out, workspace)
    _check(_lib().sol_attn3d_cross_step(_ptr(q), _shared_row_strides(q, head_dim), context.ref, _ptr(out),
                                        _shared_row_strides(out, head_dim), batch, heads, _ptr(workspace), nbytes,
                                        _stream(stream)), "sol_attn3d_cross_step")


def sol_attn3d_rope_qk(plan, q, k, q_rot, k_rot, stream=None) -> None:
    _check(_lib().sol_attn3d_rope_qk(plan, _ptr(q), _ptr(k), _ptr(q_rot), _ptr(k_rot), _stream(stream)),
           "sol_attn3d_rope_qk")


def sol_attn3d_status(plan) -> int:
    return int(_lib().sol_attn3d_status(plan))


def sol_attn3d_status_word(plan) -> int:
    w = ctypes.c_uint()
    _check(_lib().sol_attn3d_status_word(plan, ctypes.byref(w)), "sol_attn3d_status_word")
    return int(w.value)


def sol_attn3d_debug_build() -> bool:
    return bool(_lib().sol_attn3d_debug_build())


def sol_attn3d_set_profiling(plan, enable: bool) -> None:
    _check(_lib().sol_attn3d_set_profiling(plan, 1 if enable else 0), "sol_attn3d_set_profiling")


def sol_attn3d_last_forward_ms(plan) -> Tuple[float, float, float]:
    ms = (ctypes.c_float * 3)()
    _check(_lib().sol_attn3d_last_forward_ms(plan, ms), "sol_attn3d_last_forward_ms")
    return float(ms[0]), float(ms[1]), float(ms[2])


def sol_attn3d_last_launch_count(plan) -> int:
    return int(_lib().sol_attn3d_last_launch_count(plan))


def sol_attn3d_softmax_rescale_count(plan) -> int:
    n = ctypes.c_ulonglong()
    _check(_lib().sol_attn3d_softmax_rescale_count(plan, ctypes.byref(n)), "sol_attn3d_softmax_rescale_count")
    return int(n.value)


def sol_attn3d_last_cuda_error(plan) -> int:
    return int(_lib().sol_attn3d_last_cuda_error(plan))


def sol_attn3d_strerror(code: int) -> str:
    return _lib().sol_attn3d_strerror(code).decode()


def sol_attn3d_destroy(plan) -> None:
    _check(_lib().sol_attn3d_destroy(plan), "sol_attn3d_destroy")


# ----------------------------------------------------------------- convenience holder
class Attn3d:
    """Owns a plan and its torch-allocated workspace.  ``forward`` = one DiT-block attention."""

    def __init__(self, seqs, heads, head_dim, rope_dims, theta=10000.0, device="cuda", **strides):
        self.seqs = [tuple(int(x) for x in s) for s in seqs]
        self.heads, self.head_dim = heads, head_dim
        self.plan = sol_attn3d_plan_ex(self.seqs, heads, head_dim, rope_dims, theta, **strides)
        self.cu_seqlens = sol_attn3d_cu_seqlens(self.plan)
        self.total_tokens = self.cu_seqlens[-1]
        self.workspace = None
        if device is not None:
            nbytes = sol_attn3d_workspace_bytes(self.plan)
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
            assert self.workspace.data_ptr() % 256 == 0
            sol_attn3d_set_workspace(self.plan, self.workspace)

    @classmethod
    def from_workload(cls, w, device="cuda"):
        return cls([(s.text_len, s.T, s.H, s.W) for s in w.seqs], w.heads, w.head_dim, w.rope_dims, w.theta, device)

    def forward(self, q, k, v, key_mask=None, out=None, stream=None):
        if out is None:
            out = torch.empty((self.total_tokens, self.heads, self.head_dim), dtype=torch.bfloat16, device=q.device)
        sol_attn3d_forward(self.plan, q, k, v, out, key_mask, stream)
        return out

    def rope_qk(self, q, k, stream=None):
        q_rot = torch.empty((self.total_tokens, self.heads, self.head_dim), dtype=torch.bfloat16, device=q.device)
        k_rot = torch.empty_like(q_rot)
        sol_attn3d_rope_qk(self.plan, q, k, q_rot, k_rot, stream)
        return q_rot, k_rot

    def status(self) -> int:
        return sol_attn3d_status(self.plan)

    def close(self):
        if self.plan is not None:
            sol_attn3d_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
