"""After a time-out nothing is joined: the list of what to join may never have been written, or be an earlier call's."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("paged", [False, True])
def test_no_join_after_a_time_out(monkeypatch, head_dim, paged):
    """Every unit of this call has its keys split, so all rows come from the join.  The scratch still holds a healthy call's list and parts,
    all of them in range, so that a join that runs all the same shows in `out` and nowhere else."""
    from paper_2609_35110_b200 import binding as B
    dims = (16, 24, 24) if head_dim == 64 else (32, 48, 48)
    g = torch.Generator().manual_seed(1)
    n_new = 300
    q = torch.randn(n_new, 2, head_dim, generator=g).bfloat16().cuda()
    k, v = (torch.randn(1, 40, 32, 2, head_dim, generator=g).bfloat16().cuda() for _ in range(2))

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    cache = B.sol_attn3d_paged_cache(k, v, ints([list(range(40))]), ints([1280]))
    ctx = B.sol_attn3d_context(k.view(-1, 2, head_dim), v.view(-1, 2, head_dim), ints([0]), ints([1280]), 1280)
    healthy = B.Attn3d([(n_new, 0, 1, 1)], 2, head_dim, dims)
    size = B.sol_attn3d_paged_workspace_bytes(healthy.plan, cache) if paged else B.sol_attn3d_cross_workspace_bytes(healthy.plan, ctx)
    assert size > 0
    ws, out = torch.zeros(size, dtype=torch.uint8, device="cuda"), torch.empty_like(q)

    def run(attn):
        out.fill_(7.0)
        if paged:
            B.sol_attn3d_forward_paged(attn.plan, q, cache, 0, out, workspace=ws)
        else:
            B.sol_attn3d_forward_cross(attn.plan, q, ctx, out, workspace=ws)
        torch.cuda.synchronize()
        return attn.status()

    assert run(healthy) == B.OK and not bool((out == 7.0).all(-1).any())
    want = out.clone()
    assert int(ws[:4].view(torch.int32)) == 4                           # two units of rows, two heads: all of them joined
    monkeypatch.setenv("SOL_ATTN3D_WAIT_LIMIT_MS", "30")
    monkeypatch.setenv("SOL_ATTN3D_FAULT_INJECT", "1")
    broken = B.Attn3d([(n_new, 0, 1, 1)], 2, head_dim, dims)
    monkeypatch.delenv("SOL_ATTN3D_FAULT_INJECT")
    monkeypatch.delenv("SOL_ATTN3D_WAIT_LIMIT_MS")
    for _ in range(2):                                                  # the call that times out, and one behind it
        assert run(broken) == B.ERR_DEVICE_TIMEOUT and bool((out == 7.0).all())
    B.sol_attn3d_set_workspace(broken.plan, broken.workspace)           # clears the status; the hook is still in this plan
    assert run(broken) == B.ERR_DEVICE_TIMEOUT and bool((out == 7.0).all())
    assert run(healthy) == B.OK and torch.equal(out, want)
    broken.close()
    healthy.close()
