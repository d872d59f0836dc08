"""A paged cache: the pass that fills it, and forking, growing, thinning, closing of its streams and copying of its pages."""
import random

import pytest
import torch

from oracle import streaming_oracle as so

pytestmark = pytest.mark.gpu

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def rope(d):
    return (16, 24, 24) if d == 64 else (32, 48, 48)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def size(s):
    return s[0] + s[1] * s[2] * s[3]


# ---------------------------------------------------------------------------------------------- append
def rounded(out, ref, mag, slack):
    """One rounding to bf16 of a value computed in fp32.  A rotated value is a sum of two products of magnitude mag at most: the
    factors are off by 2^-24 each, products and sum by 2^-24, the norm's root by 2^-22 or so, a gain's product by 2^-24: below
    slack * mag in all."""
    bound = HALF_STEP * ref.abs() * (1 + HALF_STEP) + slack * mag + 1e-38
    bad = ~((out.double() - ref).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


def check_append(seqs, streams, lens, heads, kv, d, page, norm, pos0, eps=1e-5, dims=None, scale=1.0, q=True, gains=None, seed=0):
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(seed)
    dims = dims or rope(d)
    n = sum(size(s) for s in seqs)
    qkv = torch.randn(n, heads + 2 * kv, d, generator=g).mul(scale).bfloat16()
    n_streams = len(lens)
    counts = [-(-x // page) for x in lens]
    n_pages = sum(counts) + 2
    ids, table, at = torch.randperm(n_pages, generator=g).tolist(), torch.full((n_streams, max(counts + [1])), -1, dtype=torch.int32), 0
    for s, c in enumerate(counts):
        table[s, :c] = torch.tensor(ids[at:at + c], dtype=torch.int32)
        at += c
    pools = [torch.randn(3, n_pages, page, kv, d, generator=g).bfloat16() for _ in range(2)]
    dev = [p.cuda() for p in pools]
    cache = B.sol_attn3d_paged_cache(dev[0], dev[1], table.cuda(), ints(lens))
    x = qkv.cuda()
    attn = B.Attn3d(seqs, heads, d, dims, q_strides=(x.stride(0), d))
    q_out = torch.full((n, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    if gains is None:
        gains = [1.0 + 0.2 * torch.randn(d, generator=g) for _ in range(2)] if norm else [None, None]
    B.sol_attn3d_cache_append(attn.plan, x[:, :heads] if q else None, x[:, heads:heads + kv], x[:, heads + kv:], q_out if q else None, cache, 1,
                              streams=None if streams is None else ints(streams), pos0=None if pos0 is None else ints(pos0),
                              q_gain=None if gains[0] is None else gains[0].cuda(), k_gain=None if gains[1] is None else gains[1].cuda(), eps=eps)
    torch.cuda.synchronize()
    want = [p.double() for p in pools]
    kmag = torch.zeros_like(want[0])
    written = torch.zeros(n_pages, page, dtype=torch.bool)
    at, taken = 0, set()
    for i, s in enumerate(seqs):
        m, st = size(s), i if streams is None else streams[i]
        off = (0, 0, 0) if pos0 is None else pos0[i]
        rows = qkv[at:at + m]
        if not 0 <= st < n_streams:
            assert not q or bool((q_out[at:at + m] == 7.0).all())
        else:
            if q:
                ref = so.rotate_chunk(so.normalise(rows[:, :heads], gains[0], eps), s, dims, 10000.0, off)
                y = so.normalise(rows[:, :heads], gains[0], eps).view(m, heads, d // 2, 2).abs().sum(-1, keepdim=True).expand(-1, -1, -1, 2).reshape(m, heads, d)
                rounded(q_out[at:at + m].cpu(), ref, y, 2e-6)
            if st not in taken:
                k_ref = so.rotate_chunk(so.normalise(rows[:, heads:heads + kv], gains[1], eps), s, dims, 10000.0, off)
                y = so.normalise(rows[:, heads:heads + kv], gains[1], eps).view(m, kv, d // 2, 2).abs().sum(-1, keepdim=True).expand(-1, -1, -1, 2).reshape(m, kv, d)
                for r in range(m):
                    j = lens[st] - m + r
                    if j >= 0:
                        p = int(table[st, j // page])
                        want[0][1, p, j % page], kmag[1, p, j % page] = k_ref[r], y[r]
                        want[1][1, p, j % page] = rows[r, heads + kv:].double()
                        written[p, j % page] = True
            taken.add(st)
        at += m
    assert torch.equal(dev[1].cpu().double(), want[1])
    got = dev[0].cpu()
    rounded(got[1][written], want[0][1][written], kmag[1][written], 2e-6)
    assert torch.equal(got[1][~written].double(), want[0][1][~written])
    assert torch.equal(got[0], pools[0][0]) and torch.equal(got[2], pools[0][2])


@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (6, 2, 128), (40, 8, 128), (5, 1, 64), (1, 1, 128)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("far", [False, True])
def test_append(heads, kv, d, norm, far):
    seqs = [(3, 2, 5, 7), (0, 1, 1, 1), (9, 0, 1, 1), (1, 1, 9, 30)]
    pos0 = [[100, 3, 0], [2 ** 31 - 5, 7, 123456789], [1, 2, 3], [-4, 1 << 20, 77]] if far else None
    check_append(seqs, [2, 0, 4, 1], [1, 300, 75, 5, 64], heads, kv, d, 16 if norm else 48, norm, pos0, seed=heads)


def test_append_edges():
    """Rows before the first token, idle sequences, a stream named twice, partial rotation, no Q, one gain only."""
    check_append([(0, 1, 4, 10), (5, 0, 1, 1), (0, 1, 2, 2)], [0, -1, 7], [33, 10], 2, 1, 64, 32, True, None)
    check_append([(0, 1, 4, 10), (5, 0, 1, 1), (0, 1, 2, 2)], [1, 0, 1], [33, 50], 2, 2, 128, 16, False, [[1, 2, 3]] * 3)
    check_append([(0, 2, 3, 5)], None, [30], 3, 3, 128, 64, True, [[5, 6, 7]], dims=(20, 0, 40))
    check_append([(0, 2, 3, 5)], None, [31], 3, 3, 64, 64, True, None, q=False)
    check_append([(0, 2, 3, 5), (1, 3, 1, 1)], None, [31, 4], 1, 1, 128, 64, True, [[9, 8, 7]] * 2, q=False)
    one = torch.ones(64) * 3
    check_append([(0, 2, 3, 5)], None, [31], 3, 3, 64, 64, True, None, gains=[None, one])
    check_append([(0, 2, 3, 5)], None, [31], 3, 3, 64, 64, True, None, gains=[one, None])


@pytest.mark.parametrize("scale,eps", [(1e30, 1e-5), (1e-30, 0.0), (1e-30, 1e-5), (1e-20, 1e-38)])
def test_append_norm_keeps_its_range(scale, eps):
    """Squares outside fp32's range."""
    check_append([(1, 2, 3, 5)], None, [31], 2, 2, 128, 16, True, None, eps=eps, scale=scale)


def test_append_without_offsets_equals_the_rotary_pass():
    from paper_2609_35110_b200 import binding as B
    seqs, heads, d = [(7, 2, 6, 9)], 4, 128
    n = size(seqs[0])
    x = torch.randn(2, n, heads, d, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    attn = B.Attn3d(seqs, heads, d, rope(d))
    q_rot, k_rot = attn.rope_qk(x[0], x[1])
    pool = [torch.zeros(1, 8, 16, heads, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = B.sol_attn3d_paged_cache(pool[0], pool[1], ints([list(range(8))]), ints([n]))
    out = torch.empty_like(x[0])
    B.sol_attn3d_cache_append(attn.plan, x[0], x[1], x[1], out, cache, 0)
    assert torch.equal(out, q_rot) and torch.equal(pool[0].view(-1, heads, d)[:n], k_rot) and torch.equal(pool[1].view(-1, heads, d)[:n], x[1])


# ---------------------------------------------------------------------------------------------- bookkeeping
class Model:
    """A cache on the GPU beside its list model; every row of the pool holds numbers of its own."""

    def __init__(self, lens, page, n_pages, width, layers=2, kv=1, d=64, seed=0, interleaved=False):
        from paper_2609_35110_b200 import binding as B
        rng = random.Random(seed)
        ids, table, refs = rng.sample(range(n_pages), n_pages), [], [0] * n_pages
        for n in lens:
            c = -(-n // page)
            table.append([ids.pop() for _ in range(c)] + [-1] * (width - c))
            for p in table[-1][:c]:
                refs[p] = 1
        self.book = so.PageBook(table, lens, refs, page)
        # values name their (layer, tensor, page, row): small integers, exact in bf16
        x = torch.randint(-120, 120, (layers, n_pages, page, 2, kv, d), generator=torch.Generator().manual_seed(seed)).bfloat16()
        self.start = x
        dev = x.cuda()
        k, v = (dev[:, :, :, 0], dev[:, :, :, 1]) if interleaved else (dev[:, :, :, 0].contiguous(), dev[:, :, :, 1].contiguous())
        self.cache = B.sol_attn3d_paged_cache(k, v, ints(table), ints(lens), ints(refs))

    def ws(self, n):
        from paper_2609_35110_b200 import binding as B
        return torch.full((B.sol_attn3d_cache_workspace_bytes(self.cache, n),), 255, dtype=torch.uint8, device="cuda")

    def check(self, status=None, want=None):
        torch.cuda.synchronize()
        b, c = self.book, self.cache
        if status is not None:
            assert status.tolist() == want
        assert c.lens.tolist() == b.lens and c.refs.tolist() == b.refs and c.table.tolist() == b.table
        src = torch.tensor([[b.rows[p, r] for r in range(b.page)] for p in range(len(b.refs))])
        for i, t in enumerate((c.k, c.v)):
            assert torch.equal(t.cpu(), self.start[:, src[..., 0], src[..., 1], i])

    def call(self, what, *lists, rows=None):
        from paper_2609_35110_b200 import binding as B
        n = len(lists[0])
        status = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        if what == "reserve":
            B.sol_attn3d_cache_reserve(self.cache, ints(lists[0]), ints(lists[1]), status)
            want = self.book.reserve(*lists)
        elif what == "fork":
            B.sol_attn3d_cache_fork(self.cache, ints(lists[0]), ints(lists[1]), status, self.ws(n))
            want = self.book.fork(*lists)
        elif what == "compact":
            B.sol_attn3d_cache_compact(self.cache, ints(lists[0]), torch.tensor(lists[1], dtype=torch.uint8, device="cuda").view(n, -1), status, self.ws(n))
            want = self.book.compact(*lists)
        else:
            B.sol_attn3d_cache_free(self.cache, ints(lists[0]), status)
            want = self.book.free(lists[0])
        self.check(status, want)
        return want


@pytest.mark.parametrize("page,kv,d", [(16, 1, 64), (48, 3, 128), (128, 2, 64)])
def test_life_of_streams(page, kv, d):
    """Growing, branching, thinning and closing in turn, with requests that are refused among them."""
    m = Model([5 * page, 3 * page + 7, 0, 1, 2 * page - 1] + [0] * 5, page, 40, 12, kv=kv, d=d, seed=page, interleaved=page == 48)
    w = 12 * page
    assert m.call("fork", [0, 1, 3, 0, 2, 0], [5, 6, 7, 5, 8, -1]) == [0, 0, 0, 1, 0, 1]      # 5 is named twice, -1 is none
    assert m.call("fork", [1, 1, 99], [6, 9, 8]) == [4, 0, 1]
    assert m.call("reserve", [6, 5, 9, 2, 2, 4, 3], [page, 1, 20 * page, 0, 3, -1, 0]) == [0, 0, 2, 0, 1, 1, 0]
    keep = [[0] * w for _ in range(5)]
    for j in range(w):
        keep[0][j] = j < 10 or j > 3 * page                             # a hole
        keep[1][j] = j < 2 * page + 3                                   # a prefix that ends in a shared page
        keep[2][j] = 1                                                  # everything
        keep[3][j] = 0                                                  # nothing
        keep[4][j] = j % 3 == 1                                         # scattered
    assert m.call("compact", [5, 6, 1, 4, 0], keep) == [0] * 5
    assert m.call("free", [1, 1, 9, 50]) == [0, 1, 0, 1]
    assert m.call("compact", [6, 6], [keep[4], keep[2]]) == [0, 1]
    assert m.call("fork", [6, 8], [1, 9]) == [0, 0]
    assert m.call("free", list(range(10))) == [0] * 10
    assert set(m.book.refs) == {0} and set(m.book.lens) == {0}


def test_requests_for_more_than_there_is():
    """Sums of what is asked for pass 32 bits; nothing of it is served, what needs no page is."""
    m = Model([1, 0, 16, 5], 16, 6, 1 << 20, layers=1)
    big = (1 << 24) - 32
    from paper_2609_35110_b200 import binding as B
    n = 300
    m2 = Model([1] + [0] * n, 16, 3, 1 << 16, layers=1)
    status = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    B.sol_attn3d_cache_reserve(m2.cache, ints(list(range(1, n + 1))), ints([(1 << 20) - 5] * (n - 1) + [0]), status)
    assert status.tolist() == [3] * (n - 1) + [0]
    assert m2.cache.lens.tolist() == [1] + [0] * n and m2.cache.refs.tolist() == m2.book.refs
    assert m.call("reserve", [0, 1, 2, 3], [big, big, 0, 11]) == [3, 3, 0, 0]


@pytest.mark.parametrize("free", [0, 1, 2, 3, 5])
def test_pages_run_out(free):
    page = 16
    m = Model([20, 33, 16, 40, 0, 0, 0], page, 9 + free, 6)
    m.call("fork", [2, 0, 1], [4, 5, 6])
    m.call("reserve", [0, 1, 2, 3], [12, 17, 0, 1])
    m.call("compact", [3, 1, 0], [[0] * 30 + [1] * 66, [1] * 33 + [0] * 63, [0, 1] * 48])
    m.call("reserve", [2, 3, 0], [48, 0, 1])


def test_random_calls():
    rng = random.Random(1)
    for trial in range(12):
        page, streams, width = rng.choice([16, 32, 48]), rng.randint(1, 9), rng.randint(1, 6)
        lens = [rng.randint(0, width * page) for _ in range(streams)]
        m = Model(lens, page, sum(-(-n // page) for n in lens) + rng.randint(0, 12) + 1, width, layers=1, seed=trial)
        for _ in range(10):
            n = rng.randint(1, streams + 1)
            who = [rng.randint(-1, streams) for _ in range(n)]
            what = rng.choice(["reserve", "fork", "compact", "free"])
            if what == "reserve":
                m.call(what, who, [rng.randint(-1, 2 * page) for _ in range(n)])
            elif what == "fork":
                m.call(what, [rng.randint(-1, streams) for _ in range(n)], who)
            elif what == "compact":
                wide = rng.randint(1, width * page + 5)
                p = rng.choice([0.1, 0.5, 0.95, 1.0])
                m.call(what, who, [[int(rng.random() < p) for _ in range(wide)] for _ in range(n)])
            else:
                m.call(what, who)


def test_many_requests_and_long_streams():
    page, n = 16, 700
    m = Model([(7 * i) % 40 for i in range(n)] + [0] * n, page, 4000, 3, layers=1)
    m.call("fork", list(range(n)), list(range(n, 2 * n)))
    m.call("reserve", list(range(n, 2 * n)), [i % 9 for i in range(n)])
    m.call("free", list(range(0, n, 2)))
    rng = random.Random(2)
    m = Model([20000, 12345, 9000], 16, 4200, 1250, layers=1)
    m.call("compact", [0, 2, 1], [[int(rng.random() < 0.7) for _ in range(20000)] for _ in range(3)])


def test_copy_pages():
    from paper_2609_35110_b200 import binding as B
    m = Model([0], 48, 20, 1, layers=3, kv=3, d=128, interleaved=True)
    src, dst = [3, 7, 5, 5, -1, 2, 99, 9], [4, 8, 6, 10, 2, 20, 1, 9]
    B.sol_attn3d_cache_copy_pages(m.cache, ints(src), ints(dst))
    for a, b in ((3, 4), (7, 8), (5, 6), (5, 10)):
        for r in range(48):
            m.book.rows[b, r] = (a, r)
    m.check()


def test_captured_and_replayed():
    """One graph of closing, branching, growing and thinning, replayed: the pages come out the same every time."""
    from paper_2609_35110_b200 import binding as B
    m = Model([100, 37, 0, 0], 16, 40, 8)
    src, dst, more, status, ws = ints([0, 1]), ints([2, 3]), ints([5, 30]), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), m.ws(2)
    keep = torch.tensor([[int(j % 5 < 3) for j in range(128)]] * 2, dtype=torch.uint8, device="cuda")
    B.sol_attn3d_cache_free(m.cache, dst, status[0])                     # the first launches happen outside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sol_attn3d_cache_free(m.cache, dst, status[0])
        B.sol_attn3d_cache_fork(m.cache, src, dst, status[1], ws)
        B.sol_attn3d_cache_reserve(m.cache, dst, more, status[2])
        B.sol_attn3d_cache_compact(m.cache, dst, keep, status[3], ws)
    for _ in range(3):
        graph.replay()
        m.book.free([2, 3])
        m.book.fork([0, 1], [2, 3])
        m.book.reserve([2, 3], [5, 30])
        m.book.compact([2, 3], keep.tolist())
        m.check(status.flatten(), [0] * 8)
