"""Cross attention to an encoder's states, over a plan and one row per context, against the fp64 oracle."""
import pytest
import torch

from oracle import streaming_oracle as so
from test_gpu_paged import close, rope, size

pytestmark = pytest.mark.gpu


def contexts(lens, kv, d, seed, gap=3):
    """Contexts one after another with rows of NaN between them, in a packed tensor."""
    g = torch.Generator().manual_seed(seed)
    begins, rows = [], 0
    for n in lens:
        begins.append(rows + gap)
        rows += n + gap
    kv_t = torch.full((rows + gap, 2, kv, d), float("nan"), dtype=torch.bfloat16)
    for b, n in zip(begins, lens):
        kv_t[b:b + n] = torch.randn(n, 2, kv, d, generator=g).bfloat16()
    return kv_t, begins


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run(seqs, q, heads, d, ctx, step=False):
    from paper_2609_35110_b200 import binding as B
    out = torch.full((q.shape[0], heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    if step:
        ws = torch.full((B.sol_attn3d_cross_step_workspace_bytes(ctx, q.shape[0], heads),), 255, dtype=torch.uint8, device="cuda")
        B.sol_attn3d_cross_step(q, ctx, out, workspace=ws)
        return out.cpu()
    attn = B.Attn3d(seqs, heads, d, rope(d), q_strides=(q.stride(0), q.stride(1)))
    ws = torch.full((B.sol_attn3d_cross_workspace_bytes(attn.plan, ctx),), 255, dtype=torch.uint8, device="cuda")
    B.sol_attn3d_forward_cross(attn.plan, q, ctx, out, workspace=ws)
    torch.cuda.synchronize()
    assert attn.status() == 0
    return out.cpu()


@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (3, 3, 128), (6, 2, 128), (5, 1, 64), (40, 1, 128)])
@pytest.mark.parametrize("masked", [False, True])
def test_plan(heads, kv, d, masked):
    from paper_2609_35110_b200 import binding as B
    seqs = [(3, 2, 5, 7), (0, 1, 1, 1), (0, 2, 17, 20), (130, 0, 1, 1), (256, 0, 1, 1)]
    lens = [77, 512, 129, 0, 1]
    kv_t, begins = contexts(lens, kv, d, seed=heads)
    begins[4], lens[4] = begins[0], lens[0]                             # two sequences with one context
    g = torch.Generator().manual_seed(1)
    mask = None
    if masked:
        mask = (torch.rand(kv_t.shape[0], generator=g) < 0.6).to(torch.uint8)
        mask[begins[2]:begins[2] + lens[2]] = 0                         # nothing counts
        kv_t[begins[1]:begins[1] + 512][mask[begins[1]:begins[1] + 512] == 0] = float("inf")
    dev = kv_t.cuda()
    ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints(lens), 512, key_mask=None if mask is None else mask.cuda())
    q = torch.randn(sum(map(size, seqs)), heads + 1, d, generator=g).bfloat16()
    out = run(seqs, q.cuda()[:, :heads], heads, d, ctx)
    at = 0
    for s, b, n in zip(seqs, begins, lens):
        m = size(s)
        ref, mag = so.attend(q[at:at + m, :heads], kv_t[b:b + n, 0], kv_t[b:b + n, 1], so.key_limits(m, n, 0), None if mask is None else mask[b:b + n].bool())
        close(out[at:at + m], ref, mag)
        at += m


@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (6, 2, 128), (33, 1, 64)])
def test_step(heads, kv, d):
    from paper_2609_35110_b200 import binding as B
    lens = [1, 0, 16, 77, 1500, 300]
    kv_t, begins = contexts(lens, kv, d, seed=2)
    dev = kv_t.cuda()
    ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints(lens), 1500)
    q = torch.randn(len(lens), heads, d, generator=torch.Generator().manual_seed(3)).bfloat16()
    out = run(None, q.cuda(), heads, d, ctx, step=True)
    for i, (b, n) in enumerate(zip(begins, lens)):
        ref, mag = so.attend(q[i:i + 1], kv_t[b:b + n, 0], kv_t[b:b + n, 1], so.key_limits(1, n, 0))
        close(out[i:i + 1], ref, mag)


def test_ranges_are_clamped():
    """begins and lens outside the tensor, max_len below a length."""
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(200, 1, 64, generator=g).bfloat16() for _ in range(2))
    ctx = B.sol_attn3d_context(k.cuda(), v.cuda(), ints([-4, 150, 500, 0]), ints([150, 1000, 3, -2]), 60)
    seqs = [(140, 0, 1, 1), (2, 0, 1, 1), (3, 0, 1, 1), (1, 0, 1, 1)]
    q = torch.randn(146, 2, 64, generator=g).bfloat16()
    out = run(seqs, q.cuda(), 2, 64, ctx)
    for a, b, lo, hi in ((0, 140, 0, 150), (140, 142, 150, 200), (142, 145, 0, 0), (145, 146, 0, 0)):
        ref, mag = so.attend(q[a:b], k[lo:hi], v[lo:hi], so.key_limits(b - a, hi - lo, 0))
        close(out[a:b], ref, mag)


def test_no_states_at_all():
    from paper_2609_35110_b200 import binding as B
    empty = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    ctx = B.sol_attn3d_context(empty, empty, ints([0, 0]), ints([0, 5]), 0)
    q = torch.randn(300, 2, 64, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    assert bool((run([(299, 0, 1, 1), (1, 0, 1, 1)], q, 2, 64, ctx) == 0).all())
    assert bool((run(None, q[:2], 2, 64, ctx, step=True) == 0).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("masked", [False, True])
def test_many_sequences_most_without_states(d, masked):
    """Units without any key among units with some, more of them than are drawn ahead; fewer and more sequences than are sorted."""
    from paper_2609_35110_b200 import binding as B
    for n_seqs in (6, 32, 33, 50):
        sizes = [40, 1, 700, 300, 129, 2000][:6] + [((37 * i) % 300) + 1 for i in range(n_seqs - 6)]
        lens = [130, 5, 0, 300, 0, 0] + [0 if i % 3 else 20 + i for i in range(n_seqs - 6)]
        kv_t, begins = contexts(lens, 2, d, seed=n_seqs)
        mask = None
        if masked:
            mask = torch.ones(kv_t.shape[0], dtype=torch.uint8)
            mask[begins[0]:begins[0] + 130] = 0
            mask[begins[3]:begins[3] + 290] = 0
        dev = kv_t.cuda()
        ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints(lens), max(lens), key_mask=None if mask is None else mask.cuda())
        q = torch.randn(sum(sizes), 4, d, generator=torch.Generator().manual_seed(1)).bfloat16()
        out = run([(n, 0, 1, 1) for n in sizes], q.cuda(), 4, d, ctx)
        at = 0
        for m, b, n in zip(sizes, begins, lens):
            ref, mag = so.attend(q[at:at + m], kv_t[b:b + n, 0], kv_t[b:b + n, 1], so.key_limits(m, n, 0), None if mask is None else mask[b:b + n].bool())
            close(out[at:at + m], ref, mag)
            at += m


@pytest.mark.parametrize("heads,d", [(2, 128), (4, 64)])
def test_padded_contexts(heads, d):
    """Key tiles without a valid key, at the end, in the middle, at the start; contexts of more than 32 tiles; split keys."""
    from paper_2609_35110_b200 import binding as B
    lens = [1000, 700, 4500, 4096, 300, 130]
    kv_t, begins = contexts(lens, heads, d, seed=7)
    mask = torch.zeros(kv_t.shape[0], dtype=torch.uint8)
    for i, spans in enumerate([[(0, 100)], [(300, 301), (600, 640)], [(0, 50), (4400, 4500)], [(4095, 4096)], [], [(128, 130)]]):
        for a, b in spans:
            mask[begins[i] + a:begins[i] + b] = 1
    kv_t[mask == 0] = float("nan")
    dev = kv_t.cuda()
    ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints(lens), 4500, key_mask=mask.cuda())
    for sizes in ([300, 20, 257, 513, 40, 1], [17] * 6, [2000, 300, 1000, 128, 700, 900]):
        q = torch.randn(sum(sizes), heads, d, generator=torch.Generator().manual_seed(1)).bfloat16()
        out = run([(n, 0, 1, 1) for n in sizes], q.cuda(), heads, d, ctx)
        at = 0
        for m, b, n in zip(sizes, begins, lens):
            ref, mag = so.attend(q[at:at + m], kv_t[b:b + n, 0], kv_t[b:b + n, 1], so.key_limits(m, n, 0), mask[b:b + n].bool())
            close(out[at:at + m], ref, mag)
            at += m


def test_strided_outputs():
    """Rows of another tensor's output are left as they were, also where a sequence has no key."""
    from paper_2609_35110_b200 import binding as B
    kv_t, begins = contexts([300, 0], 2, 64, seed=3)
    dev = kv_t.cuda()
    ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints([300, 0]), 300)
    attn = B.Attn3d([(200, 0, 1, 1), (150, 0, 1, 1)], 2, 64, rope(64), out_strides=(5 * 64, 128))
    q = torch.randn(350, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16()
    buf = torch.full((350, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf.view(350, 5 * 64).as_strided((350, 2, 64), (5 * 64, 128, 1))
    ws = torch.empty(B.sol_attn3d_cross_workspace_bytes(attn.plan, ctx), dtype=torch.uint8, device="cuda")
    B.sol_attn3d_forward_cross(attn.plan, q.cuda(), ctx, buf, workspace=ws)
    torch.cuda.synchronize()
    assert attn.status() == 0
    ref, mag = so.attend(q[:200], kv_t[begins[0]:begins[0] + 300, 0], kv_t[begins[0]:begins[0] + 300, 1], so.key_limits(200, 300, 0))
    close(out[:200].cpu(), ref, mag)
    assert bool((out[200:] == 0).all()) and bool((buf[:, 1::2] == 7.0).all()) and bool((buf[:, 4] == 7.0).all())


@pytest.mark.parametrize("masked", [False, True])
def test_many_sequences_with_split_keys(masked):
    """More sequences than are planned on the device, contexts long enough to be split, empty units among the split ones."""
    from paper_2609_35110_b200 import binding as B
    sizes, lens = [(50 * i) % 299 + 1 for i in range(40)], [0 if i % 5 == 4 else 90 * i % 2000 + 1 for i in range(40)]
    for heads, kv in ((1, 1), (6, 2)):
        kv_t, begins = contexts(lens, kv, 64, seed=heads)
        g = torch.Generator().manual_seed(2)
        mask = (torch.rand(kv_t.shape[0], generator=g) < 0.7).to(torch.uint8) if masked else None
        dev = kv_t.cuda()
        ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints(lens), 2000, key_mask=None if mask is None else mask.cuda())
        q = torch.randn(sum(sizes), heads, 64, generator=g).bfloat16()
        room = torch.full((sum(sizes) + 600, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        out = room[300:300 + sum(sizes)]                                # what lies before and behind stays
        attn = B.Attn3d([(n, 0, 1, 1) for n in sizes], heads, 64, rope(64))
        ws = torch.full((B.sol_attn3d_cross_workspace_bytes(attn.plan, ctx),), 255, dtype=torch.uint8, device="cuda")
        assert ws.numel() > 0
        B.sol_attn3d_forward_cross(attn.plan, q.cuda(), ctx, out, workspace=ws)
        torch.cuda.synchronize()
        assert attn.status() == 0 and bool((room[:300] == 7.0).all()) and bool((room[300 + sum(sizes):] == 7.0).all())
        at = 0
        for m, b, n in zip(sizes, begins, lens):
            ref, mag = so.attend(q[at:at + m], kv_t[b:b + n, 0], kv_t[b:b + n, 1], so.key_limits(m, n, 0), None if mask is None else mask[b:b + n].bool())
            close(out[at:at + m].cpu(), ref, mag)
            at += m


@pytest.mark.parametrize("heads,kv", [(2, 2), (4, 2), (8, 1), (32, 1), (12, 2)])
@pytest.mark.parametrize("d,masked", [(64, True), (128, False), (128, True)])
@pytest.mark.parametrize("head_major", [False, True])
def test_whole_and_cut_tiles_at_output_strides(heads, kv, d, masked, head_major):
    """Warps whose rows are whole tokens of their sequence, and warps that a sequence's end cuts; what lies between rows stays."""
    from paper_2609_35110_b200 import binding as B
    sizes, lens = [300, 31, 1, 97, 64], [300, 0, 140, 1, 513]
    total = sum(sizes)
    kv_t, begins = contexts(lens, kv, d, seed=heads)
    g = torch.Generator().manual_seed(4)
    mask = (torch.rand(kv_t.shape[0], generator=g) < 0.7).to(torch.uint8) if masked else None
    dev = kv_t.cuda()
    ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints(begins), ints(lens), 513, key_mask=None if mask is None else mask.cuda())
    q = torch.randn(total, heads, d, generator=g).bfloat16()
    shape = (heads + 1, total + 5, d + 8) if head_major else (total + 5, heads + 1, d + 8)
    buf = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    out = (buf.transpose(0, 1) if head_major else buf)[2:2 + total, 1:, :d]
    st = out.stride()
    attn = B.Attn3d([(n, 0, 1, 1) for n in sizes], heads, d, rope(d), out_strides=st[:2])
    ws = torch.empty(B.sol_attn3d_cross_workspace_bytes(attn.plan, ctx), dtype=torch.uint8, device="cuda")
    B.sol_attn3d_forward_cross(attn.plan, q.cuda(), ctx, out, workspace=ws)
    torch.cuda.synchronize()
    assert attn.status() == 0
    at, got = 0, out.cpu()
    for m, b, n in zip(sizes, begins, lens):
        ref, mag = so.attend(q[at:at + m], kv_t[b:b + n, 0], kv_t[b:b + n, 1], so.key_limits(m, n, 0), None if mask is None else mask[b:b + n].bool())
        close(got[at:at + m], ref, mag)
        at += m
    out.fill_(7.0)
    assert bool((buf == 7.0).all())
