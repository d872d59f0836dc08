"""Differential attention over a plan keeps bf16's range of V: a power of two in V is a power of two in x."""
import pytest
import torch

from oracle import diff_linear_oracle as dlo
from test_gpu_diff import ROPE, check, make

pytestmark = pytest.mark.gpu

SEQS = [(77, 2, 9, 13), (130, 0, 1, 1), (0, 1, 1, 1)]


def forward(attn, q, k, v, w, mask=None):
    from paper_2609_35110_b200 import binding as B
    out = torch.full_like(q, 7.0)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, mask, w)
    torch.cuda.synchronize()
    assert attn.status() == 0
    return out


@pytest.mark.parametrize("exponent", [-100, -60, -40, -20, -10, 12, 20, 60, 100])
def test_powers_of_two_pass_through(exponent):
    """Without the norm everything behind the softmax is linear in V, and scaling by 2^k commutes with every rounding (no value
    leaves bf16's or fp32's normal range here): the same bits, shifted."""
    attn, (q, k, v), w, o = make(SEQS, 4, 300, gain=False)
    out = forward(attn, q, k, v, w)
    ref, cond = dlo.diff_oracle(q, k, v, SEQS, ROPE, 10000.0, **o)
    check(out, ref, cond)
    scaled = forward(attn, q, k, v * 2.0 ** exponent, w)
    assert torch.equal(scaled.float(), out.float() * 2.0 ** exponent)
    attn.close()


@pytest.mark.parametrize("eps", [0.0, 1e-5])
@pytest.mark.parametrize("exponent", [-60, -24, -17, -10, 0, 14, 40, 100])
def test_the_norm_sees_the_true_scale(exponent, eps):
    attn, (q, k, v), w, o = make(SEQS, 4, 301, gain=True, eps=eps)
    v *= 2.0 ** exponent
    out = forward(attn, q, k, v, w)
    ref, cond = dlo.diff_oracle(q, k, v, SEQS, ROPE, 10000.0, **o)
    assert float(ref.abs().max()) > 0
    up = 2.0 ** (-exponent if eps and exponent < 0 else 0)           # eps dominates there and the output is small: compare in its scale
    check(out.double() * up, ref * up, cond)
    attn.close()


def test_scales_of_sequences_and_pairs_are_their_own():
    """Every (sequence, head pair) has its own order of magnitude."""
    heads = 6
    attn, (q, k, v), w, _ = make(SEQS, heads, 302, gain=False, strided=True)
    out = forward(attn, q, k, v, w)
    cu = attn.cu_seqlens
    f = torch.ones(attn.total_tokens, heads, 1, device="cuda")
    for s in range(len(SEQS)):
        for pair in range(heads // 2):
            f[cu[s]:cu[s + 1], 2 * pair:2 * pair + 2] = 2.0 ** (25 * (s - 1) - 30 * (pair - 1))
    v2 = v.clone()
    v2.copy_(v.float() * f)
    packed = torch.stack([q, k, v2], 1).contiguous()                 # the plan's strides
    got = forward(attn, packed[:, 0], packed[:, 1], packed[:, 2], w)
    assert torch.equal(got.float(), out.float() * f)
    attn.close()


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("heads", [2, 18, 34, 74, 102, 130])
def test_many_sequences_and_head_counts(heads, masked):
    """Head counts that fill the rotary pass's blocks evenly, with an odd number of heads, with heads left over and in several goes;
    many short sequences, each (sequence, pair) with a random order of magnitude."""
    seqs = SEQS + [(3, 1, 2, 2)] * 40
    attn, (q, k, v), w, _ = make(seqs, heads, 309, gain=False)
    n = attn.total_tokens
    g = torch.Generator().manual_seed(heads)
    mask = (torch.rand(n, generator=g) < 0.7).to(torch.uint8).cuda() if masked else None
    out = forward(attn, q, k, v, w, mask)
    assert bool(torch.isfinite(out).all())
    e = torch.randint(-100, 101, (len(seqs), heads // 2), generator=g)
    lengths = torch.tensor([b - a for a, b in zip(attn.cu_seqlens, attn.cu_seqlens[1:])])
    f = (2.0 ** e.float()).repeat_interleave(lengths, 0).repeat_interleave(2, 1)[:, :, None].cuda()
    scaled = (v.float() * f).bfloat16()
    if masked:
        scaled[mask == 0] = torch.finfo(torch.bfloat16).max
    assert torch.equal(forward(attn, q, k, scaled, w, mask).float(), out.float() * f)
    attn.close()


def test_values_that_do_not_count_do_not_set_the_scale():
    attn, (q, k, v), w, _ = make(SEQS, 4, 303, gain=False)
    v *= 2.0 ** -30
    mask = torch.ones(attn.total_tokens, dtype=torch.uint8, device="cuda")
    mask[20:60] = 0
    out = forward(attn, q, k, v, w, mask)
    v[20:60] = torch.tensor([1e38, float("inf"), float("nan"), -3e38]).bfloat16().cuda().repeat(16)
    assert torch.equal(forward(attn, q, k, v, w, mask), out)
    attn.close()


def test_zero_values_and_one_large_one():
    attn, (q, k, v), w, o = make(SEQS, 2, 304, gain=False)
    v[:, :, :] = 0
    assert bool((forward(attn, q, k, v, w) == 0).all())
    v[:] = torch.randn(v.shape, generator=torch.Generator().manual_seed(1)).cuda()
    v[100, :, :] = 1e4                                               # the others are 2^-14 of it and still exact
    ref, cond = dlo.diff_oracle(q, k, v, SEQS, ROPE, 10000.0, **o)
    check(forward(attn, q, k, v, w), ref, cond)
    attn.close()


def test_replays_see_the_values_of_their_time():
    """Nothing is kept from one call for the next: a captured call, replayed with other values in the same tensors, and eager calls
    on the same plan between replays."""
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, _ = make(SEQS, 4, 305, gain=False)
    want = forward(attn, q, k, v, w)
    held, out = v.clone(), torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sol_attn3d_forward_diff(attn.plan, q, k, held, out, None, w)
    for exponent in (0, 90, -90, 3, -40, -40, 0):
        held.copy_(v * 2.0 ** exponent)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.float(), want.float() * 2.0 ** exponent), exponent
        assert torch.equal(forward(attn, q, k, v * 2.0 ** (exponent // 2), w).float(), want.float() * 2.0 ** (exponent // 2))
    attn.close()


@pytest.mark.parametrize("large", [1e4, 1e15, 1e30, 3e38])
def test_zero_rows_beside_a_large_value(large):
    """One key with a large value and a weight of exp(-512), zeros elsewhere: x is 0 and eps keeps the norm from 0 / 0."""
    attn, (q, k, v), w, o = make([(50, 0, 1, 1)], 2, 308, gain=True, eps=1e-5)
    q[..., 0], k[..., 0] = 64.0, 0.0
    k[7, :, 0] = -64.0
    v.zero_()
    v[7] = large
    assert bool((forward(attn, q, k, v, w) == 0).all())
    attn.close()


def test_a_call_that_skips_its_first_rows_counts_too():
    """Large values in a call whose query mask leaves the first blocks without work, small ones in the next."""
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, _ = make([(700, 0, 1, 1)], 2, 307, gain=False)
    out = forward(attn, q, k, v, w)
    want = torch.zeros(700, dtype=torch.uint8, device="cuda")
    for rows in (slice(0, 0), slice(600, 700)):
        want[rows] = 1
        some = torch.full_like(q, 7.0)
        B.sol_attn3d_forward_diff(attn.plan, q, k, v * 2.0 ** 100, some, None, w, want)
        sel = want.bool()
        assert torch.equal(some[sel].float(), out[sel].float() * 2.0 ** 100) and bool((some[~sel] == 7.0).all())
        small = forward(attn, q, k, v * 2.0 ** -100, w)
        assert torch.equal(small.float(), out.float() * 2.0 ** -100)
    attn.close()


@pytest.mark.parametrize("scale", [1e-7, 1e-5, 1.0, 1e6])
def test_both_forms_agree(scale):
    """The last token by the form over a plan and by the step over a cache: the first rounds Q, K and P to fp16 (a relative error of
    a map below 5e-3, the contract's), both round the output."""
    from paper_2609_35110_b200 import binding as B
    n, heads = 200, 4
    attn, (q, k, v), w, o = make([(n, 0, 1, 1)], heads, 306, gain=True, eps=0.0)
    v *= scale
    plan = forward(attn, q, k, v, w)[-1:]
    step = torch.empty_like(plan)
    lens = torch.full((1,), n, dtype=torch.int32, device="cuda")
    B.sol_attn3d_diff_step(q[-1:].contiguous(), k[None], v[None], lens, step, w, None)
    ref, cond = dlo.diff_oracle(q, k, v, [(n, 0, 1, 1)], ROPE, 10000.0, **o)
    check(plan, ref[-1:], cond[-1:])
    check(step, ref[-1:], cond[-1:])
    attn.close()
