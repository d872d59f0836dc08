"""Differential attention over a plan (sol_attn3d_forward_diff) against the fp64 oracle."""
import math

import pytest
import torch

from oracle import attn3d_oracle as orc
from oracle import diff_linear_oracle as dlo

pytestmark = pytest.mark.gpu

ROPE = (16, 24, 24)
TOL = 5e-3      # relative L2 error of one softmax map's output in the library's contract


def make(seqs, heads, seed, gain=True, eps=1e-5, per_pair=False, strided=False, lambda_init=0.35):
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(seed)
    n = sum(L + T * H * W for (L, T, H, W) in seqs)
    qkv = torch.randn(n, 3, heads, 64, generator=g).bfloat16()
    shape = (heads // 2, 64) if per_pair else (64,)
    lams = [0.15 * torch.randn(shape, generator=g) for _ in range(4)]
    gain_t = 1.0 + 0.2 * torch.randn(128, generator=g) if gain else None
    if strided:
        dev = qkv.cuda()
        q, k, v = dev[:, 0], dev[:, 1], dev[:, 2]
        st = (3 * heads * 64, 64)
        kw = dict(q_strides=st, k_strides=st, v_strides=st)
    else:
        q, k, v = (qkv[:, i].contiguous().cuda() for i in range(3))
        kw = {}
    attn = B.Attn3d(seqs, heads, 64, ROPE, **kw)
    w = B.sol_attn3d_diff_weights(*(x.cuda() for x in lams), lambda_init, None if gain_t is None else gain_t.cuda(), eps)
    lam = dlo.diff_lambda(*lams, lambda_init)
    return attn, (q, k, v), w, dict(lam=lam, lambda_init=lambda_init, gain=gain_t, eps=eps)


def check(got, ref, cond, rows=None):
    """Rows [n, heads, 64] against the oracle.  Each map's output is held to the contract's relative L2 error TOL; the
    difference amplifies a relative error by the row's condition number (the norm's derivative is a projection, which
    adds nothing), so the whole may be off by TOL times the condition-weighted norm, and a single row by 4 times that."""
    n, heads, _ = ref.shape
    err = (got.double().cpu() - ref).reshape(n, heads // 2, 128).norm(dim=-1)
    size = ref.reshape(n, heads // 2, 128).norm(dim=-1) * cond
    if rows is not None:
        err, size = err[rows], size[rows]
    assert torch.isfinite(err).all()
    assert float(err.norm()) <= TOL * float(size.norm()), (float(err.norm()) / float(size.norm()))
    assert bool((err <= 4 * TOL * size + 1e-30).all()), float((err / size.clamp(min=1e-30)).max())


@pytest.mark.parametrize("seqs, heads, kw", [
    ([(0, 4, 8, 8)], 4, {}),                                                   # the correctness grid
    ([(1, 0, 1, 1)], 2, {}),                                                   # one token
    ([(0, 1, 1, 2)], 2, dict(gain=False)),
    ([(127, 0, 1, 1)], 2, dict(per_pair=True)),
    ([(128, 0, 1, 1)], 4, dict(per_pair=True)),
    ([(129, 0, 1, 1)], 2, dict(strided=True)),
    ([(0, 3, 5, 17)], 6, dict(strided=True, per_pair=True)),                   # 255
    ([(1, 1, 16, 16)], 2, dict(gain=False)),                                   # 257
    ([(77, 5, 9, 13), (0, 1, 1, 1), (256, 4, 7, 13), (3, 1, 2, 61)], 6, dict(strided=True)),
    ([(256, 5, 9, 20)], 2, dict(eps=0.0)),
])
def test_forward_diff_matches_the_oracle(seqs, heads, kw):
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, o = make(seqs, heads, 11 + heads, **kw)
    out = torch.full((attn.total_tokens + 3, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out[:-3], None, w)
    torch.cuda.synchronize()
    assert attn.status() == 0
    ref, cond = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, **o)
    check(out[:-3], ref, cond)
    assert bool((out[-3:] == 7.0).all())                                       # rows behind the last sequence
    first = out.clone()
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out[:-3], None, w)
    assert torch.equal(out, first)
    attn.close()


@pytest.mark.parametrize("n", [2, 3, 7])
def test_maps_that_nearly_cancel(n):
    """Few keys and lambda close to 1: the norm blows up what is left of two nearly equal maps.  The output's own rounding
    aside, the error is that of the two maps (P rounded to bf16, scores from fp16 operands) times the condition number."""
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, o = make([(0, 1, 1, n)], 40, 30 + n, lambda_init=0.8)
    out = torch.empty_like(q)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
    torch.cuda.synchronize()
    ref, cond = dlo.diff_oracle(q, k, v, [(0, 1, 1, n)], ROPE, 10000.0, **o)
    check(out, ref, cond)
    attn.close()


def test_masks_empty_rows_and_query_mask():
    from paper_2609_35110_b200 import binding as B
    seqs = [(200, 3, 8, 16), (40, 2, 5, 5), (0, 1, 9, 30)]
    heads = 4
    attn, (q, k, v), w, o = make(seqs, heads, 3)
    n = attn.total_tokens
    g = torch.Generator().manual_seed(4)
    mask = (torch.rand(n, generator=g) < 0.7).to(torch.uint8)
    mask[130:300] = 0                                                          # a whole key tile and more
    mask[584:674] = 0                                                          # the second sequence has no key at all
    want = (torch.rand(n, generator=g) < 0.5).to(torch.uint8)
    want[0:256] = 0                                                            # a whole query block
    out = torch.full((n, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, mask.cuda(), w)
    torch.cuda.synchronize()
    assert attn.status() == 0
    ref, cond = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, key_mask=mask, **o)
    check(out, ref, cond)
    assert bool((out[584:674] == 0).all())
    rect = torch.full_like(out, 7.0)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, rect, mask.cuda(), w, want.cuda())
    sel = want.bool().cuda()
    assert torch.equal(rect[sel], out[sel])                                    # wanted rows: the same bits
    assert bool((rect[~sel] == 7.0).all())                                     # the others: left as they were
    # the mask of this call is not the next one's, and not the plain forward's either
    plain = attn.forward(q, k, v)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, rect, mask.cuda(), w)
    assert torch.equal(attn.forward(q, k, v), plain)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, rect, None, w)
    ref, cond = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, **o)
    check(rect, ref, cond)
    attn.close()


def test_masked_keys_do_not_matter():
    from paper_2609_35110_b200 import binding as B
    seqs = [(300, 2, 6, 6)]
    attn, (q, k, v), w, _ = make(seqs, 2, 5)
    mask = torch.ones(attn.total_tokens, dtype=torch.uint8)
    mask[100:290] = 0
    mask = mask.cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, a, mask, w)
    k[100:290] = -3.0e4
    v[100:290] = torch.finfo(torch.bfloat16).min
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, b, mask, w)
    assert torch.equal(a, b)
    attn.close()


def test_garbage_under_masks_and_in_the_neighbour_sequence():
    """Infinities and NaN in K and V at masked positions, and in the sequence that shares the last key tile, have no effect."""
    from paper_2609_35110_b200 import binding as B
    seqs = [(300, 2, 6, 6), (70, 0, 1, 1)]
    attn, (q, k, v), w, o = make(seqs, 2, 8)
    mask = torch.ones(attn.total_tokens, dtype=torch.uint8)
    mask[100:290] = 0
    for m in (mask.cuda(), None):
        off = torch.zeros(attn.total_tokens, dtype=torch.bool) if m is None else ~mask.bool()
        off[372:] = True                                                       # the second sequence's rows end the first one's tile
        a, b = torch.empty_like(q), torch.empty_like(q)
        B.sol_attn3d_forward_diff(attn.plan, q, k, v, a, m, w)
        k2, v2 = k.clone(), v.clone()
        k2[off.cuda()] = float("nan")
        v2[off.cuda()] = torch.tensor([float("nan"), float("inf")]).bfloat16().cuda().repeat(32)
        B.sol_attn3d_forward_diff(attn.plan, q, k2, v2, b, m, w)
        torch.cuda.synchronize()
        assert attn.status() == 0
        assert torch.isfinite(a).all() and torch.equal(a[:372], b[:372])
    attn.close()


def test_logit_ramp_moves_the_reference():
    """Logits that grow along the keys by far more than 2^8 per tile: both maps move their reference maximum."""
    from paper_2609_35110_b200 import binding as B
    seqs = [(640, 0, 1, 1)]
    attn, (q, k, v), w, o = make(seqs, 2, 6, gain=False)
    q[:, :, 0], k[:, :, 0] = 16.0, (torch.arange(640) // 16 * 4).to(torch.bfloat16).cuda()[:, None]
    out = torch.empty_like(q)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
    torch.cuda.synchronize()
    assert attn.status() == 0 and B.sol_attn3d_softmax_rescale_count(attn.plan) > 0
    ref, cond = dlo.diff_oracle(q, k, v, seqs, ROPE, 10000.0, **o)
    check(out, ref, cond)
    attn.close()


def test_capture_other_stream_and_two_plans():
    from paper_2609_35110_b200 import binding as B
    cases = [make([(30, 3, 7, 9)], 4, 21), make([(0, 2, 11, 13)], 2, 22, gain=False)]
    refs = [torch.empty_like(c[1][0]) for c in cases]
    for (attn, (q, k, v), w, _), r in zip(cases, refs):
        B.sol_attn3d_forward_diff(attn.plan, q, k, v, r, None, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    outs = [torch.zeros_like(r) for r in refs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for (attn, (q, k, v), w, _), r in zip(cases, outs):
            B.sol_attn3d_forward_diff(attn.plan, q, k, v, r, None, w)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs, refs):
        assert torch.equal(a, b)
    # an eager masked call between two replays changes nothing for the captured unmasked one
    attn, (q, k, v), w, _ = cases[0]
    mask = torch.zeros(attn.total_tokens, dtype=torch.uint8, device="cuda")
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, torch.empty_like(q), mask, w)
    outs[0].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], refs[0])
    late = torch.zeros_like(refs[0])
    with torch.cuda.stream(side):
        B.sol_attn3d_forward_diff(attn.plan, q, k, v, late, None, w)
    side.synchronize()
    assert torch.equal(late, refs[0])
    for c in cases:
        c[0].close()


def test_low_resolution_stage_sampled_rows():
    from paper_2609_35110_b200 import binding as B
    seqs, heads = [(256, 16, 30, 52)], 40
    attn, (q, k, v), w, o = make(seqs, heads, 9, strided=True)
    out = torch.empty(attn.total_tokens, heads, 64, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
    torch.cuda.synchronize()
    assert attn.status() == 0
    _, pos, has = orc.layout_positions(seqs)
    n = attn.total_tokens
    rows = torch.unique(torch.cat([torch.tensor([0, 255, 256, n - 1, n - 128]), torch.randint(0, n, (250,), generator=torch.Generator().manual_seed(1))]))
    for pair in (0, 7, 19):
        h = slice(2 * pair, 2 * pair + 2)
        qr, kr = (orc.rope_rotate(orc.widen(x[:, h]), pos, has, ROPE, 10000.0) for x in (q, k))
        ref, cond = dlo.diff_rows(qr[rows], kr, orc.widen(v[:, h]).reshape(n, 128), o["lam"], None, o["lambda_init"], o["gain"], o["eps"])
        check(out[rows][:, h], ref.reshape(-1, 2, 64), cond[:, None])
    attn.close()


def test_refusals():
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, _ = make([(20, 0, 1, 1)], 2, 1)
    out = torch.empty_like(q)
    with pytest.raises(ValueError):
        B.sol_attn3d_forward_diff(attn.plan, q.float(), k, v, out, None, w)
    with pytest.raises(ValueError):
        B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, torch.ones(20, device="cuda"), w)
    with pytest.raises(B.SolAttn3dError) as e:
        B.sol_attn3d_forward_diff(attn.plan, q, k, v, q, None, w)
    assert e.value.code == B.ERR_INVALID_ARG
    attn.close()


