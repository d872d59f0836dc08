"""An idle sequence of the append: nothing of it is read, neither alone nor between others."""
import pytest
import torch

from test_gpu_cache import check_append

pytestmark = pytest.mark.gpu

HBM = 8e12                        # bytes per second: no B200 reads faster from memory


def test_idle_rows_are_not_read():
    """2.1 GB of Q, K and V, seventeen times what the L2 cache holds: to read them takes 0.27 ms and more.  An idle call takes less than
    half of that, so it has not read them."""
    from paper_2609_35110_b200 import binding as B
    heads, kv, d, n = 128, 64, 128, 32768
    x = torch.zeros(n, heads + 2 * kv, d, dtype=torch.bfloat16, device="cuda")
    pool = [torch.zeros(1, 4, 16, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table, lens = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.full((1,), 64, dtype=torch.int32, device="cuda")
    cache = B.sol_attn3d_paged_cache(pool[0], pool[1], table, lens)
    attn = B.Attn3d([(0, 8, 64, 64)], heads, d, (32, 48, 48), q_strides=(x.stride(0), d))
    q_out, idle = torch.full((n, heads, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.tensor([-1], dtype=torch.int32, device="cuda")
    times = []
    for _ in range(8):
        t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        t0.record()
        B.sol_attn3d_cache_append(attn.plan, x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:], q_out, cache, 0, streams=idle)
        t1.record()
        torch.cuda.synchronize()
        times.append(t0.elapsed_time(t1) * 1e-3)
    assert min(times[3:]) < 0.5 * x.nbytes / HBM, times
    assert bool((q_out == 7.0).all())


@pytest.mark.parametrize("norm", [False, True])
def test_idle_tokens_among_others(norm):
    """Groups of neighbouring tokens (four in large plans) of which some are idle, the last group cut."""
    seqs = [(1, 0, 1, 1), (0, 1, 1, 2), (2, 0, 1, 1), (0, 1, 1, 1), (1, 1, 1, 1)] * 5 + [(0, 4, 21, 23), (3, 1, 1, 2), (0, 1, 1, 1)]
    streams = [-1 if i % 3 == 1 or i in (8, 9) else i for i in range(len(seqs))]
    streams[2], streams[-2] = 1 << 30, -5
    lens = [s[0] + s[1] * s[2] * s[3] + i for i, s in enumerate(seqs)]
    check_append(seqs, streams, lens, 6, 2, 128, 16, norm, [[i, 2 * i, 5] for i in range(len(seqs))], seed=2)
    check_append(seqs[:9], streams[:9], lens[:9], 3, 1, 64, 32, norm, None, seed=3)
