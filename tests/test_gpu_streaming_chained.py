"""Calls one right behind another give what calls one at a time give: each kernel may be on the GPU before its predecessor has written
what it reads."""
import pytest
import torch

from test_gpu_paged import rope

pytestmark = pytest.mark.gpu

HEADS, KV, D, PAGE, LAYERS, STREAMS = 8, 2, 128, 16, 2, 6


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def generate(tokens, frames, rounds, wait):
    """Token by token: streams grow, the tokens go in, every layer's query is the last one's output; then a frame of each stream, a branch of
    stream 0, a window over it.  Returns all that was written."""
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(4)
    n_pages, width = 400, 40
    zeros = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    pool = [torch.zeros(LAYERS, n_pages, PAGE, KV, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = B.sol_attn3d_paged_cache(pool[0], pool[1], zeros(STREAMS + 1, width) - 1, zeros(STREAMS + 1), zeros(n_pages))
    who, ones, framed = ints(list(range(STREAMS))), ints([1] * STREAMS), ints([frames] * STREAMS)
    plans = [B.Attn3d([(0, 1, 1, n)] * STREAMS, HEADS, D, rope(D)) for n in (1, frames)]
    scratch = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    ws_step, ws_paged = scratch(B.sol_attn3d_paged_step_workspace_bytes(cache, STREAMS, HEADS)), scratch(B.sol_attn3d_paged_workspace_bytes(plans[1].plan, cache))
    ws_book = scratch(B.sol_attn3d_cache_workspace_bytes(cache, 1))
    keep = torch.ones(1, width * PAGE, dtype=torch.uint8, device="cuda")
    keep[0, 3:9] = 0
    new = [torch.randn(rounds, LAYERS, STREAMS * n, HEADS + 2 * KV, D, generator=g, device="cuda").bfloat16() for n in (1, frames)]
    q = [torch.empty(STREAMS * n, HEADS, D, dtype=torch.bfloat16, device="cuda") for n in (1, frames)]
    x = [torch.empty_like(t) for t in q]
    pos = zeros(STREAMS, 3)
    gain, status = torch.ones(D, device="cuda"), zeros(8, STREAMS)
    seen = []

    def done():
        if wait:
            torch.cuda.synchronize()

    def one_round(r):
        for _ in range(tokens):
            B.sol_attn3d_cache_reserve(cache, who, ones, status[0])
            done()
            for layer in range(LAYERS):
                t = new[0][r, layer]
                B.sol_attn3d_cache_append(plans[0].plan, t[:, :HEADS].contiguous() if layer == 0 else x[0], t[:, HEADS:HEADS + KV], t[:, HEADS + KV:], q[0], cache, layer,
                                          pos0=pos, q_gain=gain, k_gain=gain, eps=1e-6)
                done()
                B.sol_attn3d_paged_step(q[0], cache, layer, x[0], streams=who, workspace=ws_step)
                done()
        B.sol_attn3d_cache_reserve(cache, who, framed, status[1])
        done()
        for layer in range(LAYERS):
            t = new[1][r, layer]
            B.sol_attn3d_cache_append(plans[1].plan, t[:, :HEADS].contiguous() if layer == 0 else x[1], t[:, HEADS:HEADS + KV], t[:, HEADS + KV:], q[1], cache, layer, pos0=pos)
            done()
            B.sol_attn3d_forward_paged(plans[1].plan, q[1], cache, layer, x[1], causal_block=5, workspace=ws_paged)
            done()
        B.sol_attn3d_cache_fork(cache, who[:1], ints_branch, status[2, :1], ws_book)
        done()
        B.sol_attn3d_cache_compact(cache, ints_branch, keep, status[3, :1], ws_book)
        done()
        B.sol_attn3d_paged_step(q[0][:1], cache, 1, branch_out, streams=ints_branch, workspace=ws_step)
        done()
        B.sol_attn3d_cache_free(cache, ints_branch, status[4, :1])
        done()

    ints_branch, branch_out = ints([STREAMS]), torch.empty(1, HEADS, D, dtype=torch.bfloat16, device="cuda")
    for r in range(rounds):
        one_round(r)
        seen += [x[0].clone(), x[1].clone(), branch_out.clone(), status.clone(), cache.table.clone(), cache.refs.clone(), cache.lens.clone()]
    torch.cuda.synchronize()
    assert all(p.status() == 0 for p in plans)
    assert not bool(status.any())
    return seen + pool


@pytest.mark.parametrize("frames", [2, 40])                # few rows, and tensor-core tiles
def test_chained_calls(frames):
    rounds = 480 // (8 + frames)
    want = generate(8, frames, min(rounds, 12), wait=True)
    for _ in range(4):
        got = generate(8, frames, min(rounds, 12), wait=False)
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
