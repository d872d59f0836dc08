"""The operators in one model's order: a stack that alternates linear attention and differential attention over the same
packed tensors, a clip in one call per layer, then new tokens one at a time from the carried state and cache."""
import pytest
import torch

from oracle import diff_linear_oracle as dlo

pytestmark = pytest.mark.gpu

ROPE = (0, 0, 0)                     # positions enter through the decay only: the token steps need no rotation
HEADS, D, N, NEW = 4, 64, 290, 6
DECAY = torch.log1p(-(2.0 ** -torch.linspace(1, 6, HEADS)))


def heads_of(x):
    return x.reshape(x.shape[0], HEADS, D)


def test_clip_then_tokens():
    from paper_2609_35110_b200 import binding as B
    g = torch.Generator().manual_seed(5)
    x = torch.randn(N + NEW, 3, HEADS, D, generator=g)
    x[:, 1] *= D ** -0.5
    x = x.bfloat16().cuda()
    lams = [0.15 * torch.randn(64, generator=g) for _ in range(4)]
    gain = 1.0 + 0.2 * torch.randn(128, generator=g)
    w = B.sol_attn3d_diff_weights(*(t.cuda() for t in lams), 0.3, gain.cuda(), 1e-5)
    ld = DECAY.float().cuda()
    st = (3 * HEADS * D, D)
    clip = B.Attn3d([(N, 0, 1, 1)], HEADS, D, ROPE, q_strides=st, k_strides=st, v_strides=st)

    # the clip: linear layer, its output added to the values the differential layer reads
    mixed = torch.empty(N + NEW, HEADS, D, dtype=torch.bfloat16, device="cuda")
    state = torch.empty(1, HEADS, D, D, device="cuda")
    lin_ws = torch.empty(B.sol_attn3d_linear_workspace_bytes(clip.plan), dtype=torch.uint8, device="cuda")
    q, k, v = x[:N, 0], x[:N, 1], x[:N, 2]
    B.sol_attn3d_forward_linear(clip.plan, q, k, v, mixed[:N], None, ld, 1.0, None, state, lin_ws)
    cache = torch.full((1, N + NEW, 2, HEADS, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    cache[0, :N, 0], cache[0, :N, 1] = k, v + mixed[:N]
    diff = B.Attn3d([(N, 0, 1, 1)], HEADS, D, ROPE, q_strides=st, k_strides=(2 * HEADS * D, D), v_strides=(2 * HEADS * D, D))
    out = torch.empty(N + NEW, HEADS, D, dtype=torch.bfloat16, device="cuda")
    B.sol_attn3d_forward_diff(diff.plan, q, cache[0, :N, 0], cache[0, :N, 1], out[:N], None, w)

    # new tokens: state and cache are carried on
    ws = torch.empty(B.sol_attn3d_diff_step_workspace_bytes(1, HEADS, D, N + NEW), dtype=torch.uint8, device="cuda")
    for t in range(N, N + NEW):
        B.sol_attn3d_linear_step(x[t:t + 1, 0], x[t:t + 1, 1], x[t:t + 1, 2], mixed[t:t + 1], ld, 1.0, state, state)
        cache[0, t, 0], cache[0, t, 1] = x[t, 1], x[t, 2] + mixed[t]
        lens = torch.full((1,), t + 1, dtype=torch.int32, device="cuda")
        B.sol_attn3d_diff_step(x[t:t + 1, 0], cache[:, :, 0], cache[:, :, 1], lens, out[t:t + 1], w, ws)
    torch.cuda.synchronize()
    assert clip.status() == 0 and diff.status() == 0

    # each layer against its definition on the very tensors it read
    lam = dlo.diff_lambda(*lams, 0.3)
    ref, S = dlo.linear_oracle(x[:, 0], x[:, 1], x[:, 2], [0, N + NEW], DECAY, 1.0)
    assert float((mixed.double().cpu() - ref).norm()) <= 5e-3 * float(ref.norm())
    assert float((state.double().cpu() - S).norm()) <= 2.0 ** -16 * float(S.norm())
    kk, vv = dlo.widen(cache[0, :, 0]), dlo.widen(cache[0, :, 1])
    qq = dlo.widen(x[:, 0])
    for rows, n in [(slice(0, N), N)] + [(slice(t, t + 1), t + 1) for t in range(N, N + NEW)]:
        for pair in range(HEADS // 2):
            h = slice(2 * pair, 2 * pair + 2)
            ref, cond = dlo.diff_rows(qq[rows, h], kk[:n, h], vv[:n, h].reshape(n, 128), lam, None, 0.3, gain, 1e-5)
            err = (out[rows, h].double().cpu().reshape(-1, 128) - ref).norm(dim=-1)
            size = ref.norm(dim=-1) * cond               # the maps' contract error, amplified by their difference
            assert float(err.norm()) <= 5e-3 * float(size.norm())
    clip.close()
    diff.close()
