"""fp64 CPU oracle of the differential attention and of the linear attention with decay.  TEST INFRASTRUCTURE ONLY.

Plain definitions, nothing tiled, nothing rounded; imports nothing from the package.  The rotary embedding and the
token layout are those of the dense oracle.

Differential attention, head pair i = heads (2i, 2i+1) of width d, v = [v_2i | v_2i+1] of width 2d:
    x = softmax(q~_2i k~_2i^T / sqrt(d)) v - lambda * softmax(q~_2i+1 k~_2i+1^T / sqrt(d)) v
    lambda = exp(lq1 . lk1) - exp(lq2 . lk2) + lambda_init
    out = (1 - lambda_init) * x / sqrt(mean(x^2) + eps) * gain   (no gain: out = x);  no valid key: out = 0
Linear attention, one state S [d, d] per sequence and head:
    S_t = exp(log_decay) * S_(t-1) + valid_t * k_t^T v_t,   out_t = scale * q_t S_t
"""
from __future__ import annotations

from typing import Optional, Sequence, Tuple

import torch

from .attn3d_oracle import F64, layout_positions, rope_rotate, widen


def diff_lambda(lq1, lk1, lq2, lk2, lambda_init: float) -> torch.Tensor:
    """[..., d] vectors -> lambda [...]"""
    lq1, lk1, lq2, lk2 = (widen(x) for x in (lq1, lk1, lq2, lk2))
    return torch.exp((lq1 * lk1).sum(-1)) - torch.exp((lq2 * lk2).sum(-1)) + lambda_init


def diff_rows(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam, valid: Optional[torch.Tensor], lambda_init: float = 0.0,
              gain: Optional[torch.Tensor] = None, eps: float = 0.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """One head pair: q [R, 2, d], k [N, 2, d], v [N, 2d] -> (out [R, 2d], condition [R]).

    condition = (|map 1 output| + |lambda| |map 2 output|) / |x| per row: by how much a relative error of the two maps
    grows in their difference."""
    if valid is not None:
        k, v = k[valid], v[valid]                       # masked keys take no part, whatever they hold
    if k.shape[0] == 0:
        return torch.zeros(q.shape[0], v.shape[1], dtype=F64), torch.ones(q.shape[0], dtype=F64)
    maps = []
    for m in range(2):
        s = q[:, m] @ k[:, m].T / q.shape[-1] ** 0.5
        e = torch.exp(s - s.amax(-1, keepdim=True))
        maps.append((e / e.sum(-1, keepdim=True)) @ v)
    x = maps[0] - lam * maps[1]
    norm = x.norm(dim=-1)
    cond = (maps[0].norm(dim=-1) + abs(lam) * maps[1].norm(dim=-1)) / norm.clamp(min=1e-300)
    if gain is not None:
        x = (1.0 - lambda_init) * x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * widen(gain)
    return x, cond


def diff_oracle(q, k, v, seqs: Sequence[Tuple[int, int, int, int]], rope_dims, theta, lam, key_mask=None, lambda_init=0.0,
                gain=None, eps=0.0):
    """q, k, v [total, heads, d] un-rotated; lam: one value or one per pair -> (out [total, heads, d], condition
    [total, pairs]) in fp64."""
    q, k, v = widen(q), widen(k), widen(v)
    cu, pos, has = layout_positions(seqs)
    q, k = rope_rotate(q, pos, has, rope_dims, theta), rope_rotate(k, pos, has, rope_dims, theta)
    pairs, d = q.shape[1] // 2, q.shape[2]
    lam = torch.as_tensor(lam, dtype=F64).reshape(-1).expand(pairs)
    out, cond = torch.zeros_like(q), torch.ones(q.shape[0], pairs, dtype=F64)
    for s in range(len(seqs)):
        a, b = int(cu[s]), int(cu[s + 1])
        valid = None if key_mask is None else key_mask[a:b].bool().cpu()
        for i in range(pairs):
            x, c = diff_rows(q[a:b, 2 * i: 2 * i + 2], k[a:b, 2 * i: 2 * i + 2], v[a:b, 2 * i: 2 * i + 2].reshape(b - a, 2 * d),
                             lam[i], valid, lambda_init, gain, eps)
            out[a:b, 2 * i: 2 * i + 2] = x.reshape(b - a, 2, d)
            cond[a:b, i] = c
    return out, cond


def linear_oracle(q, k, v, cu: Sequence[int], log_decay, scale: float, key_mask=None, state=None):
    """Token by token: q, k, v [total, heads, d] -> (out [total, heads, d], state [n_seqs, heads, d, d]) in fp64."""
    q, k, v = widen(q), widen(k), widen(v)
    g = torch.exp(widen(log_decay).clamp(max=0.0))[:, None, None]
    n, heads, d = len(cu) - 1, q.shape[1], q.shape[2]
    S = torch.zeros(n, heads, d, d, dtype=F64) if state is None else widen(state).clone()
    out = torch.zeros_like(q)
    for s in range(n):
        for t in range(cu[s], cu[s + 1]):
            S[s] = g * S[s]
            if key_mask is None or bool(key_mask[t]):
                S[s] += k[t][:, :, None] * v[t][:, None, :]
            out[t] = scale * (q[t][:, None, :] @ S[s])[:, 0]
    return out, S
