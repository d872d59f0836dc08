"""A decay that is NaN makes its own head NaN, in every form, and no other."""
import math

import pytest
import torch

from test_gpu_linear import make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("carry", [False, True])
@pytest.mark.parametrize("seqs", [[(5, 0, 1, 1), (40, 1, 10, 10)], [(256, 5, 30, 20)]])         # whole, and cut into pieces
def test_forward(seqs, carry, D):
    from paper_2609_35110_b200 import binding as B
    decay = torch.tensor([-0.02, -0.3, -0.1, -0.5])
    case = make(seqs, 4, D, 150, carry=carry, decay=decay.clone())
    out, dst = run(case)
    case[2][1] = math.nan
    out2, dst2 = run(case)
    assert bool(out2[:, 1].isnan().all()) and bool(dst2[:, 1].isnan().all())
    others = [0, 2, 3]
    assert torch.equal(out[:, others], out2[:, others]) and torch.equal(dst[:, others], dst2[:, others])
    q, k, v = (x[:1].contiguous() for x in case[1])
    a, b = torch.empty_like(q), torch.empty_like(q)
    s1, s2 = dst[:1].clone(), dst[:1].clone()
    B.sol_attn3d_linear_step(q, k, v, a, decay.cuda(), 1.0, s1, s1)
    B.sol_attn3d_linear_step(q, k, v, b, case[2].cuda(), 1.0, s2, s2)
    assert bool(b[:, 1].isnan().all()) and bool(s2[:, 1].isnan().all())
    assert torch.equal(a[:, others], b[:, others]) and torch.equal(s1[:, others], s2[:, others])
    case[0].close()
