"""Failure detection of the attention over contexts: a withheld signal ends in a status, not in a hang."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("n_new", [100, 300])
@pytest.mark.parametrize("paged", [False, True])
def test_withheld_signal(monkeypatch, head_dim, n_new, paged):
    from paper_2609_35110_b200 import binding as B
    dims = (16, 24, 24) if head_dim == 64 else (32, 48, 48)
    g = torch.Generator().manual_seed(1)
    q = torch.randn(n_new, 2, head_dim, generator=g).bfloat16().cuda()
    k, v = (torch.randn(1, 40, 32, 2, head_dim, generator=g).bfloat16().cuda() for _ in range(2))

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    cache = B.sol_attn3d_paged_cache(k, v, ints([list(range(40))]), ints([1280]))
    ctx = B.sol_attn3d_context(k.view(-1, 2, head_dim), v.view(-1, 2, head_dim), ints([0]), ints([1280]), 1280)
    out = torch.zeros_like(q)

    def run(attn):
        size = B.sol_attn3d_paged_workspace_bytes(attn.plan, cache) if paged else B.sol_attn3d_cross_workspace_bytes(attn.plan, ctx)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        if paged:
            B.sol_attn3d_forward_paged(attn.plan, q, cache, 0, out, workspace=ws)
        else:
            B.sol_attn3d_forward_cross(attn.plan, q, ctx, out, workspace=ws)
        torch.cuda.synchronize()
        return attn.status()

    healthy = B.Attn3d([(n_new, 0, 1, 1)], 2, head_dim, dims)
    assert run(healthy) == B.OK
    want = out.clone()
    monkeypatch.setenv("SOL_ATTN3D_WAIT_LIMIT_MS", "30")
    monkeypatch.setenv("SOL_ATTN3D_FAULT_INJECT", "1")
    broken = B.Attn3d([(n_new, 0, 1, 1)], 2, head_dim, dims)
    assert run(broken) == B.ERR_DEVICE_TIMEOUT
    assert run(broken) == B.ERR_DEVICE_TIMEOUT                          # nothing starts on a workspace with a recorded fault
    monkeypatch.delenv("SOL_ATTN3D_FAULT_INJECT")
    for _ in range(3):                                                  # the same context stays usable, and the unit counter is in order
        out.zero_()
        assert run(healthy) == B.OK and torch.equal(out, want)
    broken.close()
    healthy.close()
