"""Rows of the differential step without a valid key are zeros, whatever the weights are."""
import pytest
import torch

from test_gpu_step import check_diff, diff_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("capacity, split", [(300, False), (8192, True)])
@pytest.mark.parametrize("gain", [True, False])
@pytest.mark.parametrize("weights", ["eps 0", "infinite lambda", "both"])
def test_empty_rows_are_zeros(capacity, split, gain, weights):
    from paper_2609_35110_b200 import binding as B
    c = diff_case([0, 40, 200], 4, capacity, 200, gain=gain, mask=True)
    assert (c["ws"].numel() > 0) == split
    c["mask"][2] = 0
    eps = 0.0 if weights != "infinite lambda" else 1e-5
    lams = [x.clone() for x in c["w"].tensors[:4]]
    if weights != "eps 0":
        lams[0][:], lams[1][:] = 4.0, 4.0                                    # exp(1024)
    w = B.sol_attn3d_diff_weights(*lams, 0.35, c["w"].tensors[4], eps)
    out = torch.full((3, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_diff_step(c["q"], c["k"], c["v"], c["lens"], out, w, c["ws"], key_mask=c["mask"].cuda())
    torch.cuda.synchronize()
    assert bool((out[0] == 0).all()) and bool((out[2] == 0).all())
    if weights == "eps 0":                                                   # 1e-5 beside a mean square of 0.01 and more: see below
        normal = torch.empty_like(out)
        B.sol_attn3d_diff_step(c["q"], c["k"], c["v"], c["lens"], normal, c["w"], c["ws"], key_mask=c["mask"].cuda())
        check_diff(c, normal, 1, 1, 40)
        # the norm's change: sqrt(1 + 1e-5 / mean square) <= 1 + 5e-4, and both are rounded (2^-8 each at most)
        assert torch.allclose(out[1].float(), normal[1].float(), rtol=5e-4 + 2.0 ** -7, atol=0)


def test_empty_rows_beside_a_plan():
    """The same in the form over a plan: a sequence whose keys are all masked."""
    from paper_2609_35110_b200 import binding as B
    from test_gpu_diff import make
    attn, (q, k, v), w, _ = make([(40, 0, 1, 1), (70, 0, 1, 1)], 4, 201, eps=0.0)
    mask = torch.ones(attn.total_tokens, dtype=torch.uint8, device="cuda")
    mask[40:] = 0
    out = torch.full_like(q, 7.0)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, mask, w)
    torch.cuda.synchronize()
    assert bool((out[40:] == 0).all()) and bool(torch.isfinite(out).all()) and bool((out[:40] != 7.0).any())
    attn.close()
