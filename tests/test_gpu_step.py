"""Single-token forms: differential attention of one query over a cache, recurrent step of the linear attention."""
import gc
import math

import pytest
import torch

from oracle import diff_linear_oracle as dlo

pytestmark = pytest.mark.gpu

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module", autouse=True)
def release_cached_memory():
    """The long caches here leave gigabytes in torch's allocator, which later tests that watch the free memory would carve up."""
    yield
    gc.collect()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def diff_case(lens, heads, capacity, seed, gain=True, mask=False, n_slots=None, strided=False):
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(seed)
    batch, n_slots = len(lens), n_slots or len(lens)
    q = torch.randn(batch, heads, 64, generator=g).bfloat16()
    kv = torch.randn(n_slots, capacity, 2, heads, 64, generator=g).bfloat16()
    lams = [0.15 * torch.randn(heads // 2, 64, generator=g) for _ in range(4)]
    gain_t = 1.0 + 0.2 * torch.randn(128, generator=g) if gain else None
    key_mask = (torch.rand(n_slots, capacity, generator=g) < 0.6).to(torch.uint8) if mask else None
    dev = kv.cuda()
    k, v = (dev[:, :, 0], dev[:, :, 1]) if strided else (dev[:, :, 0].contiguous(), dev[:, :, 1].contiguous())
    w = B.sol_attn3d_diff_weights(*(x.cuda() for x in lams), 0.35, None if gain_t is None else gain_t.cuda(), 1e-5)
    ws = torch.empty(B.sol_attn3d_diff_step_workspace_bytes(batch, heads, 64, capacity), dtype=torch.uint8, device="cuda")
    return dict(q=q.cuda(), k=k, v=v, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), w=w, ws=ws, mask=key_mask,
                lam=dlo.diff_lambda(*lams, 0.35), gain=gain_t, heads=heads, capacity=capacity)


def run_diff(c, out, slots=None):
    from paper_2609_35110_b200 import binding as B
    B.sol_attn3d_diff_step(c["q"], c["k"], c["v"], c["lens"], out, c["w"], c["ws"],
                           key_mask=None if c["mask"] is None else c["mask"].cuda(), slots=slots)
    return out


def check_diff(c, out, row, slot, n):
    """One output row.  The inputs are exact, the arithmetic is fp32, the output is rounded once.  fp32: a score of 64
    products is off by at most 64 * 2^-24 * sum |q k| log2(e) / 8 (about 3e-5 here, 1e-4 at most), the exponential by
    2^-22, a sum of n / 16 terms by n / 16 * 2^-24 of the sum of magnitudes (3e-5 at 8192): 2e-4 of sum p |v| covers all."""
    for pair in range(c["heads"] // 2):
        h = slice(2 * pair, 2 * pair + 2)
        q, k = dlo.widen(c["q"][row, h])[None], dlo.widen(c["k"][slot, :n, h])
        v = dlo.widen(c["v"][slot, :n, h]).reshape(n, 128)
        valid = None if c["mask"] is None else c["mask"][slot, :n].bool()
        lam = c["lam"][pair]
        x, _ = dlo.diff_rows(q, k, v, lam, valid)
        mag, _ = dlo.diff_rows(q, k, torch.nan_to_num(v).abs(), -lam.abs(), valid)
        ref, _ = dlo.diff_rows(q, k, v, lam, valid, 0.35, c["gain"], 1e-5)
        err = 2e-4 * mag
        if c["gain"] is not None:
            rms = ((x * x).mean() + 1e-5).sqrt()
            err = 0.65 * c["gain"].double().abs() * (err + x.abs() * (err * err).mean().sqrt() / rms) / rms
        got = out[row, h].double().cpu().reshape(1, 128)
        bound = err + HALF_STEP * ref.abs() * (1 + 1e-3) + 1e-38
        assert bool(((got - ref).abs() <= bound).all()), float(((got - ref).abs() / bound).max())


@pytest.mark.parametrize("lens, heads, capacity, kw", [
    ([1], 2, 1, {}),
    ([0, 1, 2, 3], 2, 5, dict(gain=False)),
    ([63, 64, 65, 127, 128, 129, 0], 4, 129, dict(mask=True)),
    ([255, 511, 512, 513, 700], 6, 1023, dict(strided=True, mask=True, gain=False)),
    ([5000, 17, 2049, 8191], 2, 8192, dict(strided=True)),
    ([333], 8, 512, {}),
    ([7] * 150, 16, 300, dict(gain=False)),
])
def test_diff_step_matches_the_oracle(lens, heads, capacity, kw):
    c = diff_case(lens, heads, capacity, 40 + heads, **kw)
    for b, n in enumerate(lens):                                   # what lies behind a stream's last token has no effect
        c["k"][b, n:], c["v"][b, n:] = float("nan"), float("inf")
    if c["mask"] is not None:                                      # nor what lies under the mask
        off = ~c["mask"].bool().cuda()
        c["k"][off], c["v"][off] = float("inf"), float("nan")
    out = torch.full((len(lens) + 2, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    run_diff(c, out[:-2])
    torch.cuda.synchronize()
    for b, n in enumerate(lens[:12]):
        check_diff(c, out, b, b, n)
        if n == 0:
            assert bool((out[b] == 0).all())
    assert bool((out[-2:] == 7.0).all())
    first = out.clone()
    c["ws"].fill_(255)                                             # nothing is carried over in the workspace
    run_diff(c, out[:-2])
    assert torch.equal(out, first)


def test_diff_step_slots_idle_rows_and_clamped_lengths():
    c = diff_case([40, 300, 20, 300, 9, 5], 4, 300, 7, n_slots=5)
    c["lens"] = torch.tensor([40, 5000, -3, 300, 9, 5], dtype=torch.int32, device="cuda")
    slots = torch.tensor([4, 0, 1, 0, -1, 5], dtype=torch.int32, device="cuda")       # one slot twice, two idle rows
    out = torch.full((6, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    run_diff(c, out, slots)
    torch.cuda.synchronize()
    check_diff(c, out, 0, 4, 40)
    check_diff(c, out, 1, 0, 300)                                  # more than the capacity: the whole slot
    assert bool((out[2] == 0).all())
    check_diff(c, out, 3, 0, 300)
    assert bool((out[4:] == 7.0).all())


def test_diff_step_every_key_masked():
    c = diff_case([600, 600], 4, 600, 8, mask=True)
    c["mask"][0] = 0
    out = torch.full((2, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    run_diff(c, out)
    torch.cuda.synchronize()
    assert bool((out[0] == 0).all())
    check_diff(c, out, 1, 1, 600)


def test_diff_step_far_below_zero_and_far_above():
    """Scores of about -3000 and +3000: the running maximum has to follow them from the first key on."""
    for sign in (-1.0, 1.0):
        c = diff_case([100], 2, 100, 9, gain=False)
        c["q"][:, :, 0], c["k"][..., 0] = 128.0, sign * 192.0
        out = torch.empty_like(c["q"])
        run_diff(c, out)
        torch.cuda.synchronize()
        # a score of magnitude 4.4e3 (log2 domain) is off by 64 * 2^-24 * 4.5e3 = 1.7e-2 at most: too coarse for check_diff's
        # bound, fine for telling a convex mix of the values from zeros or NaN
        v = c["v"][0].double().cpu()
        ref, _ = dlo.diff_rows(dlo.widen(c["q"]), dlo.widen(c["k"][0]), v.reshape(100, 128), c["lam"][0], None)
        mag, _ = dlo.diff_rows(dlo.widen(c["q"]), dlo.widen(c["k"][0]), v.reshape(100, 128).abs(), -c["lam"][0].abs(), None)
        assert bool(((out.double().cpu().reshape(1, 128) - ref).abs() <= 0.05 * mag + HALF_STEP * ref.abs()).all())


def test_diff_step_cache_beyond_4_gib():
    """Byte offsets past 2^32: the last slot of a 5 GB cache."""
    from paper_2609_35110_b200 import binding as B
    c = diff_case([1000], 2, 1000, 10)
    n_slots, cap, heads = 5, 3_900_000, 2
    big = torch.empty(n_slots, cap, 2, heads, 64, dtype=torch.bfloat16, device="cuda")       # 9.98 GB with K and V side by side
    at = cap - 1000
    big[-1, :1000, 0], big[-1, :1000, 1] = c["k"][0], c["v"][0]
    big[-1, at:, 0], big[-1, at:, 1] = c["k"][0], c["v"][0]
    ref = run_diff(c, torch.empty_like(c["q"]))
    # the cache as one with short slots whose rows lie far apart: the last slot starts beyond 2^32 bytes
    out = torch.empty_like(ref)
    ws = torch.empty(B.sol_attn3d_diff_step_workspace_bytes(1, heads, 64, 1000), dtype=torch.uint8, device="cuda")
    slots = torch.tensor([n_slots - 1], dtype=torch.int32, device="cuda")
    for part in (slice(0, 1000), slice(at, cap)):
        B.sol_attn3d_diff_step(c["q"], big[:, part, 0], big[:, part, 1], c["lens"], out, c["w"], ws, slots=slots)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def linear_case(batch, heads, D, n_slots, seed, strided=False):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(batch, 3, heads, D, generator=g).bfloat16()
    dev = qkv.cuda()
    q, k, v = (dev[:, i] if strided else dev[:, i].contiguous() for i in range(3))
    ld = -torch.rand(heads, generator=g)
    ld[0] = 0.0
    if heads > 1:
        ld[1] = -math.inf
    state = torch.randn(n_slots, heads, D, D, generator=g)
    return q, k, v, ld, state


def ref_linear(q, k, v, ld, state, slots, scale):
    """Row by row in fp64; also the magnitudes that fp32 rounding errors are proportional to."""
    S, M = state.double().clone(), state.double().abs().clone()
    out, mag = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    q, k, v = (dlo.widen(x) for x in (q, k, v))
    g = torch.exp(ld.double().clamp(max=0))[:, None, None]
    for b, s in enumerate(slots):
        if 0 <= s < state.shape[0]:
            S[s] = g * S[s] + k[b][:, :, None] * v[b][:, None, :]
            M[s] = g * M[s] + (k[b][:, :, None] * v[b][:, None, :]).abs()
            out[b] = scale * (q[b][:, None, :] @ S[s])[:, 0]
            mag[b] = abs(scale) * (q[b].abs()[:, None, :] @ M[s])[:, 0]
    return out, mag, S, M


def check_linear(got, got_state, q, k, v, ld, state, slots, scale, tokens=1):
    """fp32 state: exp is off by 2 ulp, product and sum round once each: 2^-21 of the magnitudes per token; the output sums
    D terms in fp32 (D * 2^-24 of the magnitudes) and is rounded once."""
    out, mag, S, M = ref_linear(q, k, v, ld, state, slots, scale)
    assert bool(((got_state.double().cpu() - S).abs() <= tokens * 2.0 ** -21 * M).all())
    rows = [b for b, s in enumerate(slots) if 0 <= s < state.shape[0]]
    err = (got.double().cpu() - out).abs()[rows]
    bound = (HALF_STEP * (1 + 1e-3) * out.abs() + (tokens * 2.0 ** -21 + 128 * 2.0 ** -24) * mag)[rows]
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("batch, heads, D, strided", [(1, 1, 64, False), (1, 40, 128, True), (3, 2, 64, True), (17, 5, 128, False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_linear_step_matches_the_definition(batch, heads, D, strided, in_place):
    from paper_2609_35110_b200 import binding as B
    q, k, v, ld, state = linear_case(batch, heads, D, batch, 50 + batch, strided)
    a = state.cuda()
    b = a if in_place else torch.full_like(a, 9.0)
    out = torch.empty(batch, heads, D, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_linear_step(q, k, v, out, ld.cuda(), 0.5, a, b)
    torch.cuda.synchronize()
    check_linear(out, b, q, k, v, ld, state, list(range(batch)), 0.5)
    if not in_place:
        assert torch.equal(a.cpu(), state)


def test_linear_step_slots_idle_rows_and_repeated_slots():
    from paper_2609_35110_b200 import binding as B
    slots = [3, 6, -1, 3, 0, 7, 3, 6]                                    # slot 3 three times, 6 twice, two idle rows
    q, k, v, ld, state = linear_case(8, 3, 64, 7, 60)
    a = state.cuda()
    dst = a.clone()
    out = torch.full((8, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_linear_step(q, k, v, out, ld.cuda(), 1.0, a, dst, torch.tensor(slots, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    check_linear(out, dst, q, k, v, ld, state, slots, 1.0, tokens=3)
    assert bool((out[2] == 7.0).all()) and bool((out[5] == 7.0).all())
    for s in (1, 2, 4, 5):
        assert torch.equal(dst[s].cpu(), state[s])
    once = out.clone()
    B.sol_attn3d_linear_step(q, k, v, out, ld.cuda(), 1.0, a, a, torch.tensor(slots, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, once) and torch.equal(a, dst)               # in place: the same bits


def test_linear_step_many_rows_of_one_slot_and_graph():
    from paper_2609_35110_b200 import binding as B
    n = 300
    q, k, v, ld, state = linear_case(n, 2, 64, 1, 61)
    slots = torch.zeros(n, dtype=torch.int32, device="cuda")
    ld_dev, src, dst = ld.cuda(), state.cuda(), torch.empty_like(state, device="cuda")
    out = torch.empty(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.sol_attn3d_linear_step(q, k, v, out, ld_dev, 1.0, src, dst, slots)
    graph.replay()
    torch.cuda.synchronize()
    check_linear(out, dst, q, k, v, ld, state, [0] * n, 1.0, tokens=n)
    want = out.clone()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_step_refusals():
    from paper_2609_35110_b200 import binding as B
    c = diff_case([300] * 2, 4, 300 * 8, 1)
    assert c["ws"].numel() > 0
    out = torch.empty_like(c["q"])
    with pytest.raises(B.SolAttn3dError) as e:
        B.sol_attn3d_diff_step(c["q"], c["k"], c["v"], c["lens"], out, c["w"], None)
    assert e.value.code == B.ERR_NO_WORKSPACE
    with pytest.raises(B.SolAttn3dError) as e:
        B.sol_attn3d_diff_step(c["q"], c["k"], c["v"], c["lens"], out, c["w"], c["ws"][:-256])
    assert e.value.code == B.ERR_NO_WORKSPACE
    with pytest.raises(ValueError):
        B.sol_attn3d_diff_step(c["q"], c["k"], c["v"], c["lens"].long(), out, c["w"], c["ws"])
    with pytest.raises(ValueError):
        B.sol_attn3d_diff_step(c["q"], c["k"], c["v"][:, :5], c["lens"], out, c["w"], c["ws"])
    q, k, v, ld, state = linear_case(2, 2, 64, 1, 2)
    with pytest.raises(B.SolAttn3dError) as e:                                    # two rows, one slot, no slot numbers
        B.sol_attn3d_linear_step(q, k, v, torch.empty_like(q), ld.cuda(), 1.0, state.cuda(), state.cuda())
    assert e.value.code == B.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        B.sol_attn3d_linear_step(q, k, v, torch.empty_like(q), ld.cuda(), 1.0, state.bfloat16().cuda(), state.cuda())
