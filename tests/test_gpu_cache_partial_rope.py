"""Partial rotation in the append: dims beyond the rotated ones pass through as they are, infinities and NaN too."""
import pytest
import torch

from test_gpu_cache import ints

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("d,dims", [(128, (20, 0, 40)), (64, (16, 24, 22)), (128, (0, 0, 2)), (64, (0, 0, 0)), (128, (32, 32, 32))])
@pytest.mark.parametrize("tokens", [21, 1800])            # one token, and four, at a time
def test_what_does_not_rotate_keeps_its_bits(d, dims, tokens):
    from paper_2609_35110_b200 import binding as B
    heads, kv, page, turned = 3, 2, 16, sum(dims)
    g = torch.Generator().manual_seed(d + turned)
    x = torch.randn(tokens, heads + 2 * kv, d, generator=g).bfloat16()
    odd = x.clone()
    for i, value in enumerate((INF, -INF, NAN)):            # single values: their neighbours of the pair stay finite
        odd[i::5, :, turned + i::7] = value
    columns = (tokens - 1) // 4
    attn = B.Attn3d([(tokens - 4 * columns, 1, 4, columns)], heads, d, dims, q_strides=(x.stride(0), d))
    pages = -(-tokens // page)
    got = []
    for t in (x, odd):
        dev = t.cuda()
        pool = [torch.zeros(1, pages, page, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        cache = B.sol_attn3d_paged_cache(pool[0], pool[1], ints([list(range(pages))]), ints([tokens]))
        q_out = torch.empty(tokens, heads, d, dtype=torch.bfloat16, device="cuda")
        B.sol_attn3d_cache_append(attn.plan, dev[:, :heads], dev[:, heads:heads + kv], dev[:, heads + kv:], q_out, cache, 0, pos0=ints([[3, 50, 700]]))
        got.append(torch.cat([q_out, pool[0].view(-1, kv, d)[:tokens]], 1).cpu())
    for t, out in zip((x, odd), got):
        assert torch.equal(out[..., turned:].nan_to_num(nan=1e5), t[:, :heads + kv, turned:].nan_to_num(nan=1e5))
    assert torch.equal(got[0][..., :turned], got[1][..., :turned])
