"""Attention of new tokens over a paged cache, a chunk per stream and one token per stream, against the fp64 oracle."""
import gc

import pytest
import torch

from oracle import streaming_oracle as so

pytestmark = pytest.mark.gpu

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module", autouse=True)
def release_cached_memory():
    yield
    gc.collect()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def rope(d):
    return (16, 24, 24) if d == 64 else (32, 48, 48)


def close(out, ref, mag, slack=3e-4):
    """Elementwise.  The inputs are exact; P is rounded to bf16 for the product (half a step of every term: HALF_STEP * sum p |v|)
    and the output once (HALF_STEP of it).  fp32: a score of 128 products is off by at most 128 * 2^-24 * sum |q k| * log2(e) /
    sqrt(128), below 1e-4 for these inputs, an exponential by 2^-22, sums of n terms by far less: 3e-4 * sum p |v| covers them."""
    out = out.double()
    bound = HALF_STEP * (mag + ref.abs()) * (1 + HALF_STEP) + slack * mag + 1e-30
    bad = ~((out - ref).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), float(((out - ref).abs() / bound.clamp(min=1e-30)).nan_to_num(1e9).max()), bad.nonzero()[:4].tolist())


class Cache:
    """Streams of given lengths in a pool whose other rows are NaN, pages from all over, two layers, K and V interleaved."""

    def __init__(self, lens, page, kv_heads, d, seed, layers=2, layer=1, garbage=float("nan"), interleaved=True, width=None):
        from paper_2609_35110_b200 import binding as B
        g = torch.Generator().manual_seed(seed)
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + 3
        kv = torch.full((layers, n_pages, page, 2, kv_heads, d), garbage, dtype=torch.bfloat16)
        ids = torch.randperm(n_pages, generator=g).tolist()
        width = width or max([1] + counts) + 1
        table = torch.full((len(lens), width), -7, dtype=torch.int32)
        self.k, self.v, at = [], [], 0
        for s, (n, c) in enumerate(zip(lens, counts)):
            table[s, :c] = torch.tensor(ids[at:at + c], dtype=torch.int32)
            x = torch.randn(2, n, kv_heads, d, generator=g).bfloat16()
            self.k.append(x[0])
            self.v.append(x[1])
            for j in range(n):
                kv[layer, ids[at + j // page], j % page] = x[:, j]
            at += c
        self.layer, self.d, self.kv_heads, self.n = layer, d, kv_heads, list(lens)
        dev = kv.cuda()
        k, v = (dev[:, :, :, 0], dev[:, :, :, 1]) if interleaved else (dev[:, :, :, 0].contiguous(), dev[:, :, :, 1].contiguous())
        self.cache = B.sol_attn3d_paged_cache(k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))

    def set(self, stream, j, k=None, v=None):
        """Token j of a stream gets other contents, in the pool only."""
        page = self.cache.k.shape[2]
        p = int(self.cache.table[stream, j // page])
        for t, x in ((self.cache.k, k), (self.cache.v, v)):
            if x is not None:
                t[self.layer, p, j % page] = x


def run_chunk(seqs, streams, c, heads, q, causal=0, mask=None, out=None, stream=None):
    from paper_2609_35110_b200 import binding as B
    attn = B.Attn3d(seqs, heads, c.d, rope(c.d), q_strides=(q.stride(0), q.stride(1)))
    out = torch.full((q.shape[0], heads, c.d), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    nbytes = B.sol_attn3d_paged_workspace_bytes(attn.plan, c.cache)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    st = None if streams is None else torch.tensor(streams, dtype=torch.int32, device="cuda")
    B.sol_attn3d_forward_paged(attn.plan, q, c.cache, c.layer, out, streams=st, key_mask=mask, causal_block=causal, workspace=ws)
    torch.cuda.synchronize()
    assert attn.status() == 0
    return out.cpu()


def size(s):
    return s[0] + s[1] * s[2] * s[3]


def check_chunk(seqs, streams, c, heads, causal=0, mask=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    total = sum(size(s) for s in seqs)
    packed = torch.randn(total, heads + 3, c.d, generator=g).bfloat16()
    q = packed.cuda()[:, 1:1 + heads]
    out = run_chunk(seqs, streams, c, heads, q, causal, None if mask is None else mask.cuda())
    at = 0
    for i, s in enumerate(seqs):
        n, st = size(s), i if streams is None else streams[i]
        rows = out[at:at + n]
        if not 0 <= st < len(c.n):
            assert bool((rows == 7.0).all())
        else:
            lim = so.key_limits(n, c.n[st], causal)
            valid = None
            if mask is not None:
                valid = torch.zeros(c.n[st], dtype=torch.bool)
                m = mask[st, :c.n[st]].bool()
                valid[:len(m)] = m
            ref, mag = so.attend(packed[at:at + n, 1:1 + heads], c.k[st], c.v[st], lim, valid)
            close(rows, ref, mag)
        at += n


SHAPES = [(4, 4, 64), (3, 3, 128), (6, 2, 128), (5, 1, 64), (16, 1, 128), (40, 1, 64), (12, 4, 64)]


@pytest.mark.parametrize("heads,kv,d", SHAPES)
@pytest.mark.parametrize("page,causal", [(16, 0), (48, 1), (128, 7), (64, 100)])
def test_chunks(heads, kv, d, page, causal):
    seqs = [(0, 1, 1, 1), (3, 2, 5, 7), (0, 1, 16, 16), (130, 0, 1, 1), (1, 0, 1, 1)]
    lens = [size(seqs[4]), 73 + 128, 259, 131, 1 + 640]
    streams = [4, 1, 2, 3, 0]
    c = Cache([lens[streams.index(s)] if s != 4 else 641 for s in range(5)], page, kv, d, seed=page + heads)
    check_chunk(seqs, streams, c, heads, causal)


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 64), (2, 1, 128), (9, 3, 128)])
@pytest.mark.parametrize("causal", [0, 33])
def test_masked_streams(heads, kv, d, causal):
    """Random masks, a stream whose every key is masked, one with a single valid key far in, a mask that ends before the stream."""
    lens = [300, 257, 400, 129, 515]
    c = Cache(lens, 32, kv, d, seed=3, garbage=0.0 if causal else float("nan"))
    g = torch.Generator().manual_seed(9)
    mask = (torch.rand(5, 500, generator=g) < 0.5).to(torch.uint8)
    mask[1] = 0
    mask[2] = 0
    mask[2, 391] = 3
    if not causal:                                                      # what is masked may be anything
        for s, n in enumerate(lens):
            for j in range(0, n, 7):
                if j >= 500 or mask[s, j] == 0:
                    c.set(s, j, k=float("inf"), v=float("nan"))
    check_chunk([(0, 1, 13, 20), (200, 0, 1, 1), (10, 1, 1, 1), (0, 1, 1, 128), (0, 1, 3, 5)], None, c, heads, causal, mask)


def test_rows_before_the_stream_and_empty_streams():
    """More new tokens than the stream has: the first rows see nothing under a causal rule; empty streams; idle sequences."""
    c = Cache([0, 40, 150], 16, 2, 64, seed=5)
    seqs = [(50, 0, 1, 1), (0, 1, 9, 20), (7, 0, 1, 1), (33, 0, 1, 1)]
    for causal in (0, 1, 64):
        check_chunk(seqs, [1, 2, 0, -1], c, 4, causal)
        check_chunk(seqs, [0, 0, 3, 1 << 30], c, 2, causal)
        check_chunk(seqs, [2, 2, 2, 2], c, 6, causal)


@pytest.mark.parametrize("n_new", [1, 5, 60, 300])
@pytest.mark.parametrize("heads,kv,d", [(8, 2, 128), (2, 2, 64)])
def test_long_past(n_new, heads, kv, d):
    """Few rows over a long past: the keys are split over CTAs."""
    c = Cache([9001], 64, kv, d, seed=11, interleaved=False)
    check_chunk([(n_new, 0, 1, 1)], [0], c, heads, 0)
    check_chunk([(n_new, 0, 1, 1)], [0], c, heads, 1)


def test_scores_that_grow_and_large_values():
    """Keys whose scores rise by far more than fp32's exponent range along the stream, and values at bf16's upper end."""
    d, n = 128, 1500
    c = Cache([n], 64, 1, d, seed=2, interleaved=False)
    ramp = torch.linspace(-60.0, 60.0, n)
    for sign in (1, -1):
        for j in range(n):
            k = c.k[0][j].clone()
            k[0, 0] = sign * ramp[j]
            c.k[0][j] = k
            c.v[0][j] = c.v[0][j]
        page = 64
        for j in range(n):
            c.cache.k[c.layer, int(c.cache.table[0, j // page]), j % page] = c.k[0][j].cuda()
        g = torch.Generator().manual_seed(4)
        for n_new in (1, 200):
            q = torch.randn(n_new, 4, d, generator=g).bfloat16()
            q[..., 0] = 100.0
            out = run_chunk([(n_new, 0, 1, 1)], [0], c, 4, q.cuda())
            ref, mag = so.attend(q, c.k[0], c.v[0], so.key_limits(n_new, n, 0))
            # scores of 6000 / sqrt(128): fp32 holds them to 530 * 2^-24 * log2(e) * a few = 2e-4 of the weight
            close(out, ref, mag, slack=2e-3)


def test_infinities_and_nan_where_they_count():
    """A NaN query row is NaN and its neighbours are not; a NaN key poisons the rows that see it; an infinite value passes."""
    c = Cache([200], 16, 1, 64, seed=8)
    g = torch.Generator().manual_seed(1)
    for n_new in (2, 130):
        q = torch.randn(n_new, 1, 64, generator=g).bfloat16()
        q[1] = float("nan")
        out = run_chunk([(n_new, 0, 1, 1)], [0], c, 1, q.cuda())
        assert bool(out[1].isnan().all()) and not bool(out[0].isnan().any()) and not bool(out[2:].isnan().any())
        c.set(0, 70, v=float("inf"))
        q[1] = q[0]
        out = run_chunk([(n_new, 0, 1, 1)], [0], c, 1, q.cuda())
        assert bool((out == float("inf")).all())
        c.set(0, 70, k=float("nan"))
        out = run_chunk([(n_new, 0, 1, 1)], [0], c, 1, q.cuda())
        assert bool(out.isnan().all())
        c.set(0, 70, k=c.k[0][70].cuda(), v=c.v[0][70].cuda())


@pytest.mark.parametrize("heads,kv,d", SHAPES)
@pytest.mark.parametrize("page", [16, 80])
@pytest.mark.parametrize("masked", [False, True])
def test_step(heads, kv, d, page, masked):
    from paper_2609_35110_b200 import binding as B
    lens = [0, 1, 15, 16, 17, 128, 333, 2100]
    c = Cache(lens, page, kv, d, seed=page)
    g = torch.Generator().manual_seed(6)
    streams = [7, 3, 0, 99, 1, 2, 6, 5, 4, -1, 7]
    q = torch.randn(len(streams), heads + 1, d, generator=g).bfloat16()
    mask = (torch.rand(len(lens), 2100, generator=g) < 0.4).to(torch.uint8) if masked else None
    if masked:
        mask[5] = 0
        c.set(6, int((mask[6, :333] == 0).nonzero()[0]), k=float("nan"), v=float("inf"))
    out = torch.full((len(streams), 2, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((B.sol_attn3d_paged_step_workspace_bytes(c.cache, len(streams), heads),), 255, dtype=torch.uint8, device="cuda")
    B.sol_attn3d_paged_step(q.cuda()[:, 1:], c.cache, c.layer, out[:, 1], streams=torch.tensor(streams, dtype=torch.int32, device="cuda"),
                            key_mask=None if mask is None else mask.cuda(), workspace=ws)
    out = out.cpu()
    assert bool((out[:, 0] == 7.0).all())
    for b, s in enumerate(streams):
        if not 0 <= s < len(lens):
            assert bool((out[b, 1] == 7.0).all())
            continue
        ref, mag = so.attend(q[b:b + 1, 1:], c.k[s], c.v[s], so.key_limits(1, lens[s], 0), None if mask is None else mask[s, :lens[s]].bool())
        close(out[b:b + 1, 1], ref, mag)


def test_step_equals_a_chunk_of_one():
    from paper_2609_35110_b200 import binding as B
    c = Cache([70, 900], 16, 2, 128, seed=1)
    q = torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    out = torch.empty_like(q)
    ws = torch.empty(B.sol_attn3d_paged_step_workspace_bytes(c.cache, 2, 8), dtype=torch.uint8, device="cuda")
    B.sol_attn3d_paged_step(q, c.cache, 1, out, workspace=ws)
    both = run_chunk([(1, 0, 1, 1)] * 2, None, c, 8, q)
    for s, n in enumerate(c.n):
        ref, mag = so.attend(q[s:s + 1].cpu(), c.k[s], c.v[s], so.key_limits(1, n, 0))
        close(out[s:s + 1].cpu(), ref, mag)
        close(both[s:s + 1], ref, mag)


def test_bad_pages_read_as_zeros():
    """Entries of the table that name no page, and lengths out of range."""
    from paper_2609_35110_b200 import binding as B
    for n_new in (1, 140):
        c = Cache([400], 32, 1, 64, seed=3, width=13)
        c.cache.table[0, 2] = -1
        c.cache.table[0, 5] = 1 << 20
        k, v = c.k[0].clone(), c.v[0].clone()
        for page in (2, 5):
            k[32 * page:32 * page + 32] = 0
            v[32 * page:32 * page + 32] = 0
        q = torch.randn(n_new, 2, 64, generator=torch.Generator().manual_seed(n_new)).bfloat16()
        out = run_chunk([(n_new, 0, 1, 1)], [0], c, 2, q.cuda())
        ref, mag = so.attend(q, k, v, so.key_limits(n_new, 400, 0))
        close(out, ref, mag)
        c.cache.lens[0] = -5
        assert bool((run_chunk([(n_new, 0, 1, 1)], [0], c, 2, q.cuda()) == 0).all())


def test_captured_and_replayed():
    """A captured call follows the lengths, tables and streams as they are when it is replayed."""
    from paper_2609_35110_b200 import binding as B
    c = Cache([500, 2000, 37], 16, 2, 64, seed=21)
    seqs, heads = [(0, 1, 10, 20), (1, 0, 1, 1)], 4
    attn = B.Attn3d(seqs, heads, 64, rope(64))
    q = torch.randn(201, heads, 64, generator=torch.Generator().manual_seed(5)).bfloat16()
    dq, out, streams = q.cuda(), torch.zeros(201, heads, 64, dtype=torch.bfloat16, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ws = torch.empty(B.sol_attn3d_paged_workspace_bytes(attn.plan, c.cache), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.sol_attn3d_forward_paged(attn.plan, dq, c.cache, 1, out, streams=streams, causal_block=50, workspace=ws)
    for order in ([0, 1], [1, 2], [2, 0]):
        streams.copy_(torch.tensor(order, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for (a, b), s in zip(((0, 200), (200, 201)), order):
            ref, mag = so.attend(q[a:b], c.k[s], c.v[s], so.key_limits(b - a, c.n[s], 50))
            close(out[a:b].cpu(), ref, mag)


@pytest.mark.parametrize("n_new", [1, 200])
def test_pages_beyond_4_gib(n_new):
    from paper_2609_35110_b200 import binding as B
    page, kv, d = 64, 4, 128
    n_pages = (1 << 32) // (page * kv * d * 2) + 50                     # K and V of 4 GiB and more each
    k, v = (torch.empty(1, n_pages, page, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = [n_pages - 1, 0, n_pages - 3, n_pages - 2]
    g = torch.Generator().manual_seed(7)
    kr, vr = (torch.randn(4 * page, kv, d, generator=g).bfloat16() for _ in range(2))
    for i, p in enumerate(ids):
        k[0, p], v[0, p] = kr[i * page:(i + 1) * page].cuda(), vr[i * page:(i + 1) * page].cuda()
    c = Cache([1], 16, kv, d, seed=0)
    c.cache = B.sol_attn3d_paged_cache(k, v, torch.tensor([ids], dtype=torch.int32, device="cuda"), torch.tensor([250], dtype=torch.int32, device="cuda"))
    c.layer = 0
    q = torch.randn(n_new, kv, d, generator=g).bfloat16()
    out = run_chunk([(n_new, 0, 1, 1)], [0], c, kv, q.cuda())
    ref, mag = so.attend(q, kr[:250], vr[:250], so.key_limits(n_new, 250, 0))
    close(out, ref, mag)


def test_many_streams_with_split_keys():
    """A whole wave of units and a rest whose keys are split; some streams empty, some idle, rows that see nothing."""
    lens = [4000, 0, 2500, 700, 3000, 20]
    seqs = [(700, 0, 1, 1), (40, 0, 1, 1), (300, 0, 1, 1), (130, 0, 1, 1), (1, 0, 1, 1), (100, 0, 1, 1), (257, 0, 1, 1)]
    for heads, kv, d in ((24, 24, 64), (30, 6, 128), (3, 1, 64)):
        c = Cache(lens, 32, kv, d, seed=heads, layers=1, layer=0)
        check_chunk(seqs, [2, 1, 0, 9, 4, 5, 3], c, heads, 0)
        check_chunk(seqs, [2, 1, 0, 9, 4, 5, 3], c, heads, 130)


@pytest.mark.parametrize("heads,kv", [(130, 1), (300, 2)])
def test_more_heads_per_key_head_than_a_tile_has_rows(heads, kv):
    c = Cache([500, 90], 32, kv, 64, seed=1)
    check_chunk([(20, 0, 1, 1), (1, 0, 1, 1)], None, c, heads, 1)


@pytest.mark.parametrize("heads,kv,d", [(15, 1, 128), (5, 1, 64), (40, 2, 128)])
@pytest.mark.parametrize("longest", [900, 12000])
def test_step_joins_few_and_many_parts(heads, kv, d, longest):
    """Few parts are joined by a warp per row, many by four: idle and empty streams, one without a valid key, units of 16 and of 4 rows."""
    from paper_2609_35110_b200 import binding as B
    lens = [longest, 0, longest // 3, 700, 1]
    c = Cache(lens, 64, kv, d, seed=heads)
    g = torch.Generator().manual_seed(8)
    mask = (torch.rand(5, longest, generator=g) < 0.7).to(torch.uint8)
    mask[3] = 0
    mask[4] = 1
    streams = [2, 1, 9, 0, 3, 4]
    q = torch.randn(len(streams), heads, d, generator=g).bfloat16()
    out = torch.full((len(streams), heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    nbytes = B.sol_attn3d_paged_step_workspace_bytes(c.cache, len(streams), heads)
    units = len(streams) * -(-heads // kv // 16) * kv
    assert (nbytes > units * 8 * 16 * (d + 4) * 4 + 256) == (longest > 900)          # more than 8 parts, or not
    B.sol_attn3d_paged_step(q.cuda(), c.cache, c.layer, out, streams=torch.tensor(streams, dtype=torch.int32, device="cuda"), key_mask=mask.cuda(),
                            workspace=torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda"))
    out = out.cpu()
    for b, s in enumerate(streams):
        if s >= len(lens):
            assert bool((out[b] == 7.0).all())
            continue
        ref, mag = so.attend(q[b:b + 1], c.k[s], c.v[s], so.key_limits(1, lens[s], 0), mask[s, :lens[s]].bool())
        close(out[b:b + 1], ref, mag)


def test_the_binding_refuses_masks_without_columns_and_plans_from_elsewhere():
    from paper_2609_35110_b200 import binding as B
    c = Cache([40], 16, 2, 64, seed=0)
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    nothing = torch.zeros(1, 0, dtype=torch.uint8, device="cuda")
    attn = B.Attn3d([(3, 0, 1, 1)], 2, 64, rope(64))
    with pytest.raises(ValueError):
        B.sol_attn3d_forward_paged(attn.plan, q, c.cache, 0, out, key_mask=nothing)
    with pytest.raises(ValueError):
        B.sol_attn3d_paged_step(q[:1], c.cache, 0, out[:1], key_mask=nothing)
    one = torch.tensor([0], dtype=torch.int32, device="cuda")
    x = torch.zeros(40, 2, 64, dtype=torch.bfloat16, device="cuda")
    context = B.sol_attn3d_context(x, x, one, one, 1)
    kv = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert attn.plan.device == torch.cuda.current_device()
    attn.plan.device += 1                                               # as if its workspace had been bound there
    for call in (lambda: B.sol_attn3d_forward_paged(attn.plan, q, c.cache, 0, out), lambda: B.sol_attn3d_forward_cross(attn.plan, q, context, out),
                 lambda: B.sol_attn3d_cache_append(attn.plan, None, kv, kv, None, c.cache, 0)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
