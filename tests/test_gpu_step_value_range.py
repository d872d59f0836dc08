"""The differential step's norm where the squares of the values leave fp32's range."""
import pytest
import torch

from test_gpu_step import diff_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("capacity", [300, 8192])
@pytest.mark.parametrize("exponent", [-100, -80, -50, 50, 80, 100])
def test_norm_of_small_and_large_values(capacity, exponent):
    """eps = 0: the norm takes a factor 2^k out again.  Sums of products scale exactly; what is left are the norm's own fp32
    roundings (a few 2^-24, whichever way the sum of squares is formed) and the output's, which may fall either way: one step."""
    from paper_2609_35110_b200 import binding as B
    c = diff_case([40, 250, capacity], 4, capacity, 210)
    w = B.sol_attn3d_diff_weights(*c["w"].tensors[:4], 0.35, c["w"].tensors[4], 0.0)
    plain = B.sol_attn3d_diff_weights(*c["w"].tensors[:4], 0.35, None, 0.0)

    def step(v, weights):
        out = torch.full_like(c["q"], 7.0)
        B.sol_attn3d_diff_step(c["q"], c["k"], v, c["lens"], out, weights, c["ws"])
        return out.float()

    scaled = c["v"] * 2.0 ** exponent
    assert torch.equal(step(scaled, plain), step(c["v"], plain) * 2.0 ** exponent)
    a, b = step(c["v"], w), step(scaled, w)
    assert bool(torch.isfinite(a).all()) and torch.allclose(a, b, rtol=2.0 ** -7, atol=0)
