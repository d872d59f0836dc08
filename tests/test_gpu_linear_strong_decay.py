"""Linear attention over a plan with strong finite decays: what is left is the token itself, and its weight is exactly 1."""
import pytest
import torch

from test_gpu_linear import HALF_STEP, check, make, run

pytestmark = pytest.mark.gpu

DECAYS = torch.tensor([-40.0, -100.0, -300.0, -1000.0, -3000.0, -6900.0, -6932.0, -1e6])
SEQS = {"whole": [(70, 2, 9, 11), (0, 1, 1, 130)], "cut": [(256, 5, 30, 20)]}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", ["whole", "cut"])
def test_the_token_itself_counts_once(shape, D):
    """<q, k> = 1 and scale = 1: a token's own score is 1, which bf16 holds, so P V is v itself.  What comes before has a weight
    of at most exp(-40) = 4e-18 on scores of 1 and values of at most 2: far below half a bf16 step of |v| >= 1."""
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), ld, _, ws = make(SEQS[shape], len(DECAYS), D, 140, carry=False, decay=DECAYS)
    q.zero_()
    k.zero_()
    q[..., 3], k[..., 3] = 1.0, 1.0
    v.copy_(torch.where(v < 0, -1.0, 1.0) * (1.0 + v.abs().clamp(max=0.99)))
    out, dst = run((attn, (q, k, v), ld, None, ws))
    for h in range(len(DECAYS)):
        assert torch.equal(out[:, h], v[:, h]), (float(DECAYS[h]), float((out[:, h].float() / v[:, h].float() - 1).abs().max()))
    # the recurrent form, from the state that the last but one token would have left
    step = torch.empty_like(v[-1:])
    state = torch.zeros(1, len(DECAYS), D, D, device="cuda")
    B.sol_attn3d_linear_step(q[-1:], k[-1:], v[-1:], step, ld.cuda(), 1.0, state, state)
    assert torch.equal(step, v[-1:])
    attn.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", ["whole", "cut"])
def test_random_scores_under_strong_decays(shape, D):
    """The output is scale <q, k> v: P is rounded once, the output once (HALF_STEP each, on the value), the score sums D products
    in fp32 (D * 2^-24 of their magnitudes), and so do the earlier tokens, whose weight is below 5e-18."""
    case = make(SEQS[shape], len(DECAYS), D, 141, decay=DECAYS)
    out, dst = run(case, 0.75)
    check(case, out, dst, 0.75)
    _, (q, k, v), _, _, _ = case
    q, k, v = (x.double() for x in (q, k, v))
    ref = 0.75 * (q * k).sum(-1, keepdim=True) * v
    mag = 0.75 * (q * k).abs().sum(-1, keepdim=True) * v.abs()
    bound = (2 * HALF_STEP + HALF_STEP ** 2 + 2.0 ** -20) * ref.abs() + (D + 8) * 2.0 ** -24 * mag + 1e-14
    err = (out.double() - ref).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    case[0].close()


@pytest.mark.parametrize("D", [64, 128])
def test_decays_between(D):
    """Decays from weak to strong, as the recurrence has them."""
    decay = torch.tensor([-0.003, -0.1, -1.0, -4.0, -12.0, -20.0, -87.0, -104.0])
    case = make([(30, 1, 9, 11), (0, 1, 1, 257)], 8, D, 142, decay=decay)
    out, dst = run(case, 1.0)
    check(case, out, dst, 1.0)
    case[0].close()
