"""Failure detection in the differential and the linear attention: a test hook makes one CTA withhold a signal (nothing
faults, traps or spins forever); the waits that depend on it run into their limit, the kernels return, the status word
reports the time-out, and the plan works again once the word is cleared."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def hooked_plan(monkeypatch, seqs, heads, D, rope):
    from paper_2609_35110_b200 import binding as B
    monkeypatch.setenv("SOL_ATTN3D_WAIT_LIMIT_MS", "20")
    monkeypatch.setenv("SOL_ATTN3D_FAULT_INJECT", "1")
    bad = B.Attn3d(seqs, heads, D, rope)                    # the plan reads the two variables when it is built
    monkeypatch.delenv("SOL_ATTN3D_FAULT_INJECT")
    monkeypatch.delenv("SOL_ATTN3D_WAIT_LIMIT_MS")
    return bad


def timed_out(bad, call):
    from paper_2609_35110_b200 import binding as B
    t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    t0.record()
    call(bad.plan)
    t1.record()
    torch.cuda.synchronize()                                # returns: no wait is unbounded
    assert t0.elapsed_time(t1) < 2000.0
    assert bad.status() == B.ERR_DEVICE_TIMEOUT
    call(bad.plan)                                          # refused at the door by every CTA until the word is cleared
    torch.cuda.synchronize()
    assert bad.status() == B.ERR_DEVICE_TIMEOUT
    B.sol_attn3d_set_workspace(bad.plan, bad.workspace)
    assert bad.status() == 0
    bad.close()


def tensors(n, heads, D, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, heads, D, generator=g).bfloat16().cuda() for _ in range(3)]


@pytest.mark.parametrize("gain", [True, False])
def test_differential_attention(monkeypatch, gain):
    from paper_2609_35110_b200 import binding as B
    seqs = [(40, 3, 9, 20), (0, 1, 5, 5)]
    bad = hooked_plan(monkeypatch, seqs, 4, 64, (16, 24, 24))
    q, k, v = tensors(bad.total_tokens, 4, 64, 1)
    w = B.sol_attn3d_diff_weights(*(0.1 * torch.ones(64, device="cuda") for _ in range(4)), 0.5,
                                  torch.ones(128, device="cuda") if gain else None)
    out, ref = torch.empty_like(q), torch.empty_like(q)
    timed_out(bad, lambda plan: B.sol_attn3d_forward_diff(plan, q, k, v, out, None, w))
    good = B.Attn3d(seqs, 4, 64, (16, 24, 24))              # same process, same context
    B.sol_attn3d_forward_diff(good.plan, q, k, v, ref, None, w)
    torch.cuda.synchronize()
    assert good.status() == 0 and torch.isfinite(ref).all()
    good.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs, cut", [([(1, 0, 1, 1)], False), ([(0, 1, 1, 300)] * 200, False), ([(256, 5, 30, 20)], True)])
def test_linear_attention(monkeypatch, seqs, cut, D):
    from paper_2609_35110_b200 import binding as B
    rope = (16, 24, 24) if D == 64 else (32, 48, 48)
    bad = hooked_plan(monkeypatch, seqs, 3, D, rope)
    q, k, v = tensors(bad.total_tokens, 3, D, 2)
    ld = torch.full((3,), -0.01, device="cuda")
    ws = torch.empty(B.sol_attn3d_linear_workspace_bytes(bad.plan), dtype=torch.uint8, device="cuda")
    assert (ws.numel() > 0) == cut
    out = torch.empty_like(q)
    timed_out(bad, lambda plan: B.sol_attn3d_forward_linear(plan, q, k, v, out, None, ld, 1.0, None, None, ws))
    good = B.Attn3d(seqs, 3, D, rope)
    B.sol_attn3d_forward_linear(good.plan, q, k, v, out, None, ld, 1.0, None, None, ws)
    torch.cuda.synchronize()
    assert good.status() == 0 and torch.isfinite(out).all()
    good.close()
