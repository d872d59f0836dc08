"""Pins of the differential-attention and linear-attention oracles: special cases, closed forms, brute force."""
import math

import torch

from oracle import attn3d_oracle as orc
from oracle import diff_linear_oracle as dlo

F64 = torch.float64
ROPE = (16, 24, 24)


def _inputs(n, heads, d, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, heads, d, generator=g, dtype=F64) for _ in range(3)]


def test_diff_with_lambda_zero_is_the_dense_attention_of_the_first_map():
    seqs = [(3, 2, 2, 3), (0, 1, 2, 2)]
    q, k, v = _inputs(19, 4, 64, 1)
    out, cond = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, 0.0)
    for pair in range(2):
        for half in range(2):
            h = 2 * pair + half                       # the dense attention of head 2*pair's maps over head h's values
            ref = orc.attn3d_oracle(q[:, 2 * pair:2 * pair + 1], k[:, 2 * pair:2 * pair + 1], v[:, h:h + 1], seqs, ROPE, 10000.0)
            torch.testing.assert_close(out[:, h:h + 1], ref, rtol=1e-12, atol=1e-13)
    assert torch.allclose(cond, torch.ones_like(cond))


def test_diff_of_uniform_maps_is_one_minus_lambda_times_the_mean_and_the_norm_has_unit_rms():
    seqs = [(2, 1, 1, 5)]
    _, k, v = _inputs(7, 2, 64, 2)
    q = torch.zeros(7, 2, 64, dtype=F64)
    out, _ = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, 0.3)
    mean = v.mean(0, keepdim=True).expand(7, 2, 64)
    torch.testing.assert_close(out, 0.7 * mean, rtol=1e-12, atol=1e-13)
    normed, _ = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, 0.3, lambda_init=0.25, gain=torch.full((128,), 2.0))
    x = normed.reshape(7, 128)
    torch.testing.assert_close((x * x).mean(-1).sqrt(), torch.full((7,), 1.5, dtype=F64))
    torch.testing.assert_close(x / x.norm(dim=-1, keepdim=True), (mean / mean.reshape(7, 128).norm(dim=-1)[0]).reshape(7, 128))


def test_diff_lambda_and_masks():
    a = torch.full((64,), 0.125)
    lam = dlo.diff_lambda(a, a, 2 * a, -a, 0.2)
    assert abs(float(lam) - (math.exp(1.0) - math.exp(-2.0) + 0.2)) < 1e-12
    seqs = [(4, 0, 1, 1)]
    q, k, v = _inputs(4, 2, 64, 3)
    v[1], k[1] = float("inf"), float("nan")                    # masked: whatever they hold
    mask = torch.tensor([1, 0, 1, 1])
    out, _ = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, 0.5, mask)
    keep = [0, 2, 3]
    ref, _ = dlo.diff_rows(q, k[keep], v[keep].reshape(3, 128), 0.5, None)
    torch.testing.assert_close(out.reshape(4, 128), ref)
    zero, _ = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, 0.5, torch.zeros(4))
    assert bool((zero == 0).all())


def test_linear_against_the_double_sum():
    q, k, v = _inputs(11, 2, 8, 4)
    ld = torch.tensor([-0.3, 0.0], dtype=F64)
    state = torch.randn(2, 2, 8, 8, generator=torch.Generator().manual_seed(5), dtype=F64)
    mask = torch.ones(11)
    mask[2] = 0
    cu = [0, 4, 11]
    out, S = dlo.linear_oracle(q, k, v, cu, ld, 0.7, mask, state)
    for s in range(2):
        for h in range(2):
            for i in range(cu[s], cu[s + 1]):
                n = i - cu[s] + 1
                ref = math.exp(float(ld[h]) * n) * (q[i, h] @ state[s, h])
                for j in range(cu[s], i + 1):
                    if mask[j]:
                        ref = ref + math.exp(float(ld[h]) * (i - j)) * (q[i, h] @ k[j, h]) * v[j, h]
                torch.testing.assert_close(out[i, h], 0.7 * ref)


def test_linear_carries_its_state_and_forgets_at_log_decay_minus_infinity():
    q, k, v = _inputs(9, 1, 8, 6)
    ld = torch.tensor([-0.1], dtype=F64)
    whole, S = dlo.linear_oracle(q, k, v, [0, 9], ld, 1.0)
    a, Sa = dlo.linear_oracle(q[:5], k[:5], v[:5], [0, 5], ld, 1.0)
    b, Sb = dlo.linear_oracle(q[5:], k[5:], v[5:], [0, 4], ld, 1.0, state=Sa)
    torch.testing.assert_close(torch.cat([a, b]), whole)
    torch.testing.assert_close(Sb, S)
    now, _ = dlo.linear_oracle(q, k, v, [0, 9], torch.tensor([-math.inf]), 1.0)
    torch.testing.assert_close(now, (q * k).sum(-1, keepdim=True) * v)          # only the token itself is left
