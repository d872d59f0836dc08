"""The split of a weighted key into two bf16 parts, hi + lo: seen alone when one key is all that a state holds."""
import math

import pytest
import torch

from test_gpu_linear import make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs", [[(77, 0, 1, 1)], [(128, 0, 1, 1)], [(256, 5, 30, 20)]])
@pytest.mark.parametrize("masked", [True, False])
def test_state_of_a_single_key(seqs, D, masked):
    """One key that is not masked (or not zero), values of 1: the state is w k with w a power of the decay.

    w = wb + wc + r and k wb = hi + d: every rounding to bf16 is off by at most HALF_STEP = 2^-8 of what is rounded.
        |w - wb| <= 2^-8 |w|, so |r| <= 2^-16 |w|;                     |d| <= 2^-8 |k wb|, its rounding 2^-16 |k wb|;
        lo = rn(k wc + rn(d)), at most 2 * 2^-8 |k w| (1 + 2^-7), so its rounding is at most 2^-15 |k w| (1 + 2^-7).
    Together 2^-14 |k w| (1 + 2^-6).  w itself comes out of fp32: 2^-20 covers exp2 and the products of the table."""
    heads = 8
    decay = torch.tensor([math.log(0.5292931), -0.01, -0.3, -0.05, -0.7, -0.123, -0.0004, -0.2])
    attn, (q, k, v), ld, _, ws = make(seqs, heads, D, 160, carry=False, decay=decay)
    n = attn.total_tokens
    at = n - 2
    mask = torch.zeros(n, dtype=torch.uint8)
    mask[at] = 1
    v.fill_(1.0)
    k[at, :, 0] = 1.0703125
    if not masked:
        k *= mask.cuda()[:, None, None]
    _, dst = run((attn, (q, k, v), ld, None, ws), 1.0, mask if masked else None)
    ref = torch.exp(ld.double())[:, None, None] * k[at].double().cpu()[:, :, None].expand(heads, D, D)
    err = ((dst[0].double().cpu() - ref) / ref).abs()
    assert float(err.max()) <= 2.0 ** -14 * (1 + 2.0 ** -6) + 2.0 ** -20, float(err.max()) * 2 ** 16
    attn.close()
