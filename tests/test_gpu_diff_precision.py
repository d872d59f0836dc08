"""Precision of the differential attention over a plan, and its largest size."""
import pytest
import torch

from oracle import attn3d_oracle as orc
from oracle import diff_linear_oracle as dlo
from test_gpu_diff import ROPE, check, make

pytestmark = pytest.mark.gpu


def test_error_is_the_outputs_own_rounding():
    """Random inputs, well conditioned.  Rounding the output to bf16 is a relative error of 2^-8 / sqrt(3), uniform in a binade: 0.0015
    to 0.0017 of the 2-norm, depending on how the values lie in their binades.  fp16 operands add 2^-11 / sqrt(3) = 0.0003 in
    P and, through the scores, in Q and K, in quadrature and times the condition number (1.3 here): below 0.0021 with room.
    P rounded to bf16 instead (0.0015 * 1.3) would be at 0.0024 or more, bf16 Q and K above that."""
    seqs, heads = [(256, 4, 13, 20)], 8
    for gain in (False, True):
        attn, (q, k, v), w, o = make(seqs, heads, 320, gain=gain)
        from paper_2609_35110_b200 import binding as B
        out = torch.empty_like(q)
        B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
        torch.cuda.synchronize()
        ref, _ = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, **o)
        err = float((out.double().cpu() - ref).norm() / ref.norm())
        assert err <= 0.0021, err
        attn.close()


def test_high_resolution_stage_sampled_rows():
    from paper_2609_35110_b200 import binding as B
    seqs, heads = [(256, 31, 45, 80)], 4
    attn, (q, k, v), w, o = make(seqs, heads, 321, strided=True)
    n = attn.total_tokens
    out = torch.empty(n, heads, 64, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
    torch.cuda.synchronize()
    assert attn.status() == 0 and n == 111856
    _, pos, has = orc.layout_positions(seqs)
    rows = torch.unique(torch.cat([torch.tensor([0, 255, 256, n - 1, n - 128]),
                                   torch.randint(0, n, (60,), generator=torch.Generator().manual_seed(2))]))
    for pair in range(heads // 2):
        h = slice(2 * pair, 2 * pair + 2)
        qr, kr = (orc.rope_rotate(orc.widen(x[:, h]), pos, has, ROPE, 10000.0) for x in (q, k))
        ref, cond = dlo.diff_rows(qr[rows], kr, orc.widen(v[:, h]).reshape(n, 128), o["lam"], None, o["lambda_init"], o["gain"], o["eps"])
        check(out[rows][:, h], ref.reshape(-1, 2, 64), cond[:, None])
    attn.close()
