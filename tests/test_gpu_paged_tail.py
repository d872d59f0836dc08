"""Units of one kind, more than a wave of them: whole ones in a whole wave, the keys of the rest split and joined."""
import pytest
import torch

from oracle import streaming_oracle as so
from test_gpu_paged import Cache, close, rope

pytestmark = pytest.mark.gpu

KV, KEYS, SMS = 80, 2000, 148


def joined(ws):
    """How many units the call has joined (the list's length stands first in its workspace)."""
    return int(ws[:4].view(torch.int32))


def check(out, q, sizes, keys, limits, valid=None):
    at = 0
    for i, n in enumerate(sizes):
        ref, mag = so.attend(q[at:at + n], *keys(i), limits(n), None if valid is None else valid(i))
        close(out[at:at + n], ref, mag)
        at += n


@pytest.mark.parametrize("sizes,group", [([300], 1), ([150, 150], 1), ([150], 2)])
@pytest.mark.parametrize("causal", [0, 33])
@pytest.mark.parametrize("masked", [False, True])
def test_paged(sizes, group, causal, masked):
    """160 units of 16 key tiles."""
    from paper_2609_35110_b200 import binding as B
    c = Cache([KEYS] * len(sizes), 64, KV, 64, seed=3, layers=1, layer=0, garbage=0.0)
    heads = KV * group
    g = torch.Generator().manual_seed(5)
    q = torch.randn(sum(sizes), heads, 64, generator=g).bfloat16()
    mask = (torch.rand(len(sizes), KEYS, generator=g) < 0.7).to(torch.uint8) if masked else None
    attn = B.Attn3d([(n, 0, 1, 1) for n in sizes], heads, 64, rope(64))
    out = torch.full_like(q, 7.0, device="cuda")
    ws = torch.full((B.sol_attn3d_paged_workspace_bytes(attn.plan, c.cache),), 255, dtype=torch.uint8, device="cuda")
    B.sol_attn3d_forward_paged(attn.plan, q.cuda(), c.cache, 0, out, key_mask=None if mask is None else mask.cuda(), causal_block=causal, workspace=ws)
    torch.cuda.synchronize()
    assert attn.status() == 0 and B.sol_attn3d_last_launch_count(attn.plan) == 2 and joined(ws) == 160 - SMS
    check(out.cpu(), q, sizes, lambda i: (c.k[i], c.v[i]), lambda n: so.key_limits(n, KEYS, causal), None if mask is None else lambda i: mask[i].bool())


@pytest.mark.parametrize("masked", [False, True])
def test_contexts(masked):
    """Two sequences with one context; rows written by boxes beside joined ones."""
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(6)
    sizes = [150, 129]
    kv = torch.randn(KEYS, 2, KV, 64, generator=g).bfloat16()
    q = torch.randn(sum(sizes), KV, 64, generator=g).bfloat16()
    mask = (torch.rand(KEYS, generator=g) < 0.7).to(torch.uint8) if masked else None
    dev = kv.cuda()

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    ctx = B.sol_attn3d_context(dev[:, 0], dev[:, 1], ints([0, 0]), ints([KEYS, KEYS]), KEYS, key_mask=None if mask is None else mask.cuda())
    attn = B.Attn3d([(n, 0, 1, 1) for n in sizes], KV, 64, rope(64))
    out = torch.full_like(q, 7.0, device="cuda")
    ws = torch.full((B.sol_attn3d_cross_workspace_bytes(attn.plan, ctx),), 255, dtype=torch.uint8, device="cuda")
    B.sol_attn3d_forward_cross(attn.plan, q.cuda(), ctx, out, workspace=ws)
    torch.cuda.synchronize()
    assert attn.status() == 0 and joined(ws) == 160 - SMS
    check(out.cpu(), q, sizes, lambda i: (kv[:, 0], kv[:, 1]), lambda n: so.key_limits(n, KEYS, 0), None if mask is None else lambda i: mask.bool())
