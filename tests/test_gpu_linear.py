"""Linear attention with a decay per head over a plan (sol_attn3d_forward_linear) against the fp64 recurrence."""
import math

import pytest
import torch

from oracle import diff_linear_oracle as dlo

pytestmark = pytest.mark.gpu

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2       # 2^-8: P, the state's copy for the tensor core and the output are rounded to bf16


def rope_dims(D):
    return (16, 24, 24) if D == 64 else (32, 48, 48)


def make(seqs, heads, D, seed, strided=False, carry=True, decay=None):
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(seed)
    n = sum(L + T * H * W for (L, T, H, W) in seqs)
    qkv = torch.randn(n, 3, heads, D, generator=g)
    qkv[:, 1] *= D ** -0.5
    dev = qkv.bfloat16().cuda()
    kw = {}
    if strided:
        st = (3 * heads * D, D)
        kw = dict(q_strides=st, k_strides=st, v_strides=st)
    q, k, v = (dev[:, i] if strided else dev[:, i].contiguous() for i in range(3))
    attn = B.Attn3d(seqs, heads, D, rope_dims(D), **kw)
    ld = decay if decay is not None else torch.log1p(-(2.0 ** -torch.linspace(1, 9, heads))) if heads > 1 else torch.tensor([-0.05])
    state = torch.randn(len(seqs), heads, D, D, generator=g) if carry else None
    ws = torch.empty(B.sol_attn3d_linear_workspace_bytes(attn.plan), dtype=torch.uint8, device="cuda")
    return attn, (q, k, v), ld.float(), state, ws


def run(case, scale=1.0, mask=None, out=None, state_out=True, in_place=False):
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), ld, state, ws = case
    heads, D = q.shape[1:]
    out = torch.full((attn.total_tokens, heads, D), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    src = None if state is None else state.cuda()
    dst = (src if in_place else torch.full((len(attn.seqs), heads, D, D), 9.0, device="cuda")) if state_out else None
    B.sol_attn3d_forward_linear(attn.plan, q, k, v, out, None if mask is None else mask.cuda(), ld.cuda(), scale, src, dst, ws)
    torch.cuda.synchronize()
    assert attn.status() == 0
    return out, dst


def magnitudes(q, k, v, cu, ld, scale, mask, state):
    """The same recurrence on absolute values: what the absolute error of a term-wise rounded evaluation is proportional to."""
    def dense(x):
        return torch.nan_to_num(dlo.widen(x)).abs()
    return dlo.linear_oracle(dense(q), dense(k), dense(v), cu, ld, abs(scale), mask, None if state is None else state.abs())


def check(case, got, got_state, scale=1.0, mask=None, tokens=None):
    """State: every term is a product of exact bf16 values with a power of the decay, held as hi + lo bf16 (2^-16 relative at
    worst: half a step of a half step) and summed in fp32 (128 terms per tile, then one fma per tile: n / 128 more roundings):
    (2^-16 + (256 + n / 128) * 2^-24) of the magnitudes.  Output: P and the state's copy are rounded to bf16 (half a step each, on the
    magnitudes), the sum once more (on the value), fp32 elsewhere."""
    attn, (q, k, v), ld, state, _ = case
    cu = attn.cu_seqlens
    kk, vv = k, v
    if mask is not None:                                     # the oracle drops masked keys; keep what they hold out of 0 * x
        off = ~mask.bool().cuda()
        kk, vv = k.clone(), v.clone()
        kk[off], vv[off] = 0, 0
    ref, S = dlo.linear_oracle(q, kk, vv, cu, ld, scale, mask, state)
    mag, M = magnitudes(q, kk, vv, cu, ld, scale, mask, state)
    n = max(b - a for a, b in zip(cu, cu[1:]))
    fp32 = (256 + n / 128) * 2.0 ** -24
    err, bound = (got.double().cpu() - ref).abs(), HALF_STEP * 1.01 * ref.abs() + (HALF_STEP + 2.0 ** -15 + 2 * fp32) * mag + 1e-30
    assert bool((err <= bound).all()), float((err / bound).max())
    # independent roundings do not all point the same way: in the 2-norm the whole is held to the contract's 5e-3
    assert float((got.double().cpu() - ref).norm()) <= 5e-3 * float(ref.norm()) + 1e-30
    if got_state is not None:
        err, bound = (got_state.double().cpu() - S).abs(), (2.0 ** -16 + fp32) * M + 1e-37
        assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs, heads, kw", [
    ([(1, 0, 1, 1)], 1, {}),
    ([(0, 1, 1, 2)], 2, dict(carry=False)),
    ([(127, 0, 1, 1)], 2, {}),
    ([(128, 0, 1, 1)], 3, dict(strided=True)),
    ([(129, 0, 1, 1)], 2, dict(strided=True, carry=False)),
    ([(0, 4, 8, 8)], 4, {}),
    ([(3, 2, 9, 21), (0, 1, 1, 1), (200, 2, 5, 11), (64, 0, 1, 1)], 3, dict(strided=True)),
    ([(256, 4, 7, 13)], 40, dict(strided=True)),
    ([(40, 3, 9, 11), (5, 1, 20, 20)], 5, dict(strided=True)),
])
def test_forward_linear_matches_the_recurrence(seqs, heads, kw, D):
    case = make(seqs, heads, D, 70 + heads, **kw)
    out, dst = run(case, 0.75)
    check(case, out, dst, 0.75)
    again, dst2 = run(case, 0.75)
    assert torch.equal(out, again) and torch.equal(dst, dst2)
    case[0].close()


@pytest.mark.parametrize("D", [64, 128])
def test_long_sequence_in_pieces(D):
    """Long enough, with few heads, to be cut: pieces start from the states of their predecessors."""
    from paper_2609_35110_b200 import binding as B
    seqs = [(256, 5, 30, 20), (100, 2, 30, 20)]
    decay = torch.tensor([0.0, -2.0 ** -11, -0.02, -math.inf])
    case = make(seqs, 4, D, 80, strided=True, decay=decay)
    assert B.sol_attn3d_linear_workspace_bytes(case[0].plan) > 0
    mask = (torch.rand(case[0].total_tokens, generator=torch.Generator().manual_seed(1)) < 0.8).to(torch.uint8)
    for m in (None, mask):
        out, dst = run(case, 1.0, m)
        check(case, out, dst, 1.0, m)
    case[4].fill_(255)                                        # nothing is carried over in the scratch
    inp, dst_in = run(case, 1.0, mask, in_place=True)
    assert torch.equal(inp, out) and torch.equal(dst_in, dst)
    no_state, _ = run(case, 1.0, mask, state_out=False)
    assert torch.equal(no_state, out)
    case[0].close()
    odd = make([(17, 7, 20, 20)], 3, D, 81, strided=True)       # an odd number of heads, cut
    out, dst = run(odd)
    check(odd, out, dst)
    odd[0].close()


@pytest.mark.parametrize("D", [64, 128])
def test_masks_and_garbage_under_them(D):
    seqs = [(150, 2, 8, 16), (30, 1, 5, 5)]
    case = make(seqs, 2, D, 90)
    attn, (q, k, v), ld, state, ws = case
    mask = (torch.rand(attn.total_tokens, generator=torch.Generator().manual_seed(2)) < 0.6).to(torch.uint8)
    mask[120:300] = 0                                         # a whole tile and more
    mask[attn.cu_seqlens[1]:] = 0                             # the second sequence: only its initial state is left
    out, dst = run(case, 1.0, mask)
    check(case, out, dst, 1.0, mask)
    off = ~mask.bool().cuda()
    k[off], v[off] = float("nan"), float("inf")
    out2, dst2 = run(case, 1.0, mask)
    assert torch.equal(out, out2) and torch.equal(dst, dst2)
    attn.close()


def test_decays_from_none_to_everything_and_clamped():
    D, heads = 64, 6
    decay = torch.tensor([0.0, 0.7, -1e-6, -0.5, -30.0, -math.inf])      # 0.7 counts as 0
    case = make([(0, 3, 10, 11), (77, 1, 6, 10)], heads, D, 91, decay=decay)
    out, dst = run(case, 1.0)
    check(case, out, dst, 1.0)
    assert torch.equal(out[:, 5].isnan(), torch.zeros_like(out[:, 5], dtype=torch.bool))
    case[0].close()


def test_neighbouring_sequences_and_rows_behind_the_last_do_not_leak():
    seqs = [(100, 0, 1, 1), (30, 0, 1, 1)]
    case = make(seqs, 2, 128, 92)
    attn, (q, k, v), ld, state, ws = case
    out = torch.full((attn.total_tokens + 200, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    a, _ = run(case, 1.0, out=out[:-200])
    assert bool((out[-200:] == 7.0).all())
    first = a[:100].clone()
    for x in (q, k, v):
        x[100:] = float("nan")                                # the tile of the first sequence reads into the second one
    b, dst = run(case, 1.0)
    assert torch.equal(b[:100], first) and bool(torch.isfinite(dst[0]).all())
    attn.close()


@pytest.mark.parametrize("D", [64, 128])
def test_chunked_and_recurrent_forms_continue_each_other(D):
    """A clip in one call, then token by token from its state, against all tokens in one call: states to fp32, outputs to bf16."""
    from paper_2609_35110_b200 import binding as B
    heads, n, extra = 3, 300, 5
    whole = make([(n + extra, 0, 1, 1)], heads, D, 93, carry=False)
    ref, ref_state = run(whole)
    check(whole, ref, ref_state)
    _, (q, k, v), ld, _, _ = whole
    part = B.Attn3d([(n, 0, 1, 1)], heads, D, rope_dims(D))
    ws = torch.empty(B.sol_attn3d_linear_workspace_bytes(part.plan), dtype=torch.uint8, device="cuda")
    out = torch.empty(n + extra, heads, D, dtype=torch.bfloat16, device="cuda")
    state = torch.empty(1, heads, D, D, device="cuda")
    ld_dev = ld.cuda()
    B.sol_attn3d_forward_linear(part.plan, q[:n], k[:n], v[:n], out[:n], None, ld_dev, 1.0, None, state, ws)
    for t in range(n, n + extra):
        B.sol_attn3d_linear_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], out[t:t + 1], ld_dev, 1.0, state, state)
    torch.cuda.synchronize()
    check(whole, out, state)
    whole[0].close()
    part.close()


def test_capture_streams_and_scratch_of_two_graphs():
    from paper_2609_35110_b200 import binding as B
    cases = [make([(0, 6, 20, 20)], 2, 128, 94), make([(0, 6, 20, 20)], 2, 128, 95)]
    lds = [c[2].cuda() for c in cases]
    srcs = [c[3].cuda() for c in cases]
    refs = [run(c) for c in cases]
    side = torch.cuda.Stream()
    outs = [torch.zeros_like(r[0]) for r in refs]
    dsts = [torch.zeros_like(r[1]) for r in refs]
    ws = cases[0][4]
    assert ws.numel() > 0
    graphs = []
    for i, (attn, (q, k, v), _, _, _) in enumerate(cases):    # both graphs use the first case's scratch, one after the other
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            B.sol_attn3d_forward_linear(attn.plan, q, k, v, outs[i], None, lds[i], 1.0, srcs[i], dsts[i], ws)
    for _ in range(2):
        for gr in graphs:
            gr.replay()
    torch.cuda.synchronize()
    for o, d, r in zip(outs, dsts, refs):
        assert torch.equal(o, r[0]) and torch.equal(d, r[1])
    for c in cases:
        c[0].close()


def test_high_resolution_stage_first_and_last_tokens():
    """111,856 tokens x 40 heads x 128: the first tokens against the recurrence, the last ones against a sum over the window
    that the decay leaves, and the state."""
    seqs, heads, D = [(256, 31, 45, 80)], 40, 128
    case = make(seqs, heads, D, 96, strided=True, decay=torch.full((40,), -0.01))
    attn, (q, k, v), ld, state, ws = case
    out, dst = run(case)
    n = attn.total_tokens
    for h in (0, 23, 39):
        sub = slice(h, h + 1)
        ref, _ = dlo.linear_oracle(q[:400, sub], k[:400, sub], v[:400, sub], [0, 400], ld[sub], 1.0, None, state[:, sub])
        assert float((out[:400, sub].double().cpu() - ref).norm()) <= 5e-3 * float(ref.norm())
        a = n - 4000                                          # exp(-0.01 * 3600) = 2e-16: what came before does not matter
        ref, S = dlo.linear_oracle(q[a:, sub], k[a:, sub], v[a:, sub], [0, 4000], ld[sub], 1.0)
        assert float((out[a + 3600:, sub].double().cpu() - ref[3600:]).norm()) <= 5e-3 * float(ref[3600:].norm())
        assert float((dst[0, sub].double().cpu() - S[0]).norm()) <= 2.0 ** -16 * float(S.norm())
    attn.close()


def test_refusals():
    from paper_2609_35110_b200 import binding as B
    case = make([(0, 6, 20, 20)], 2, 64, 97)
    attn, (q, k, v), ld, state, ws = case
    out, d = torch.empty_like(q), ld.cuda()
    for bad in (None, ws[:-256]):
        with pytest.raises(B.SolAttn3dError) as e:
            B.sol_attn3d_forward_linear(attn.plan, q, k, v, out, None, d, 1.0, None, None, bad)
        assert e.value.code == B.ERR_NO_WORKSPACE
    with pytest.raises(ValueError):
        B.sol_attn3d_forward_linear(attn.plan, q, k, v, out, None, ld, 1.0, None, None, ws)
    with pytest.raises(ValueError):
        B.sol_attn3d_forward_linear(attn.plan, q, k, v, out, None, d, 1.0, state.half().cuda(), None, ws)
    with pytest.raises(B.SolAttn3dError):
        B.sol_attn3d_forward_linear(attn.plan, q, k, v, v, None, d, 1.0, None, None, ws)
    attn.close()


@pytest.mark.parametrize("seqs, heads, D", [
    ([(5, 2, 4, 4)] * 700 + [(128, 8, 12, 12)], 3, 64),        # one long sequence that is cut, many short ones behind it
    ([(1, 0, 1, 1)] * 1500, 1, 128),                           # single tokens
    ([(0, 1, 1, 300)] * 3 + [(64, 9, 10, 12)] * 2, 2, 128),
])
def test_many_sequences(seqs, heads, D):
    case = make(seqs, heads, D, 130)
    out, dst = run(case, 0.5)
    check(case, out, dst, 0.5)


def test_states_of_another_number_of_sequences_are_refused():
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), ld, state, ws = make([(5, 0, 1, 1), (9, 0, 1, 1)], 2, 64, 131)
    out = torch.empty_like(q)
    for a, b in ((state[:1], None), (None, state[:1]), (state, torch.cat([state, state]))):
        a, b = (None if x is None else x.cuda() for x in (a, b))
        with pytest.raises(ValueError):
            B.sol_attn3d_forward_linear(attn.plan, q, k, v, out, None, ld.cuda(), 1.0, a, b, ws)
    attn.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs", [[(5, 0, 1, 1)], [(256, 5, 30, 20)]])         # whole, and cut into pieces
def test_a_decay_of_zero_forgets_a_state_that_holds_anything(seqs, D):
    from paper_2609_35110_b200 import binding as B
    decay = torch.tensor([-math.inf, -0.02])
    case = make(seqs, 2, D, 132, decay=decay)
    out, dst = run(case)
    check(case, out, dst)
    attn, qkv, ld, state, ws = case
    state[:, 0] = torch.tensor([math.nan, math.inf]).repeat(D // 2)
    out2, dst2 = run(case)
    assert torch.equal(out, out2) and torch.equal(dst, dst2)
    # one more token
    q, k, v = (x[:1].contiguous() for x in qkv)
    a, b = torch.empty_like(q), torch.empty_like(q)
    s1, s2 = state.cuda(), torch.nan_to_num(state, posinf=0.0).cuda()
    B.sol_attn3d_linear_step(q, k, v, a, ld.cuda(), 1.0, s1, s1)
    B.sol_attn3d_linear_step(q, k, v, b, ld.cuda(), 1.0, s2, s2)
    assert torch.equal(a, b) and torch.equal(s1, s2) and torch.isfinite(s1).all()
    attn.close()


def test_profiling_and_launch_count():
    """Per-kernel times are those of the most recent call, the linear one included."""
    from paper_2609_35110_b200 import binding as B
    for seqs, launches in (([(5, 0, 1, 1)], 1), ([(256, 5, 30, 20)], 2)):
        case = make(seqs, 2, 64, 133)
        attn, (q, k, v) = case[:2]
        ref, _ = run(case)
        B.sol_attn3d_set_profiling(attn.plan, True)
        with pytest.raises(B.SolAttn3dError):
            B.sol_attn3d_last_forward_ms(attn.plan)
        out, _ = run(case)
        assert B.sol_attn3d_last_launch_count(attn.plan) == launches
        ms = B.sol_attn3d_last_forward_ms(attn.plan)
        assert ms[0] == 0 and 0 <= ms[1] < ms[2]
        assert torch.equal(out, ref)
        attn.close()
