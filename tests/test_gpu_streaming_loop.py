"""The streaming operators together, as a generator uses them: streams grow chunk by chunk over all layers of a small stack, attend to
their past and to a prompt, branch, drop what lies outside a window and go on token by token."""
import pytest
import torch

from oracle import streaming_oracle as so
from test_gpu_paged import close, rope

pytestmark = pytest.mark.gpu

LAYERS, HEADS, KV, D, PAGE = 2, 6, 2, 64, 16
EPS = 1e-6


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Loop:
    def __init__(self, n_streams=4, n_pages=90, width=24):
        from paper_2609_35110_b200 import binding as B
        self.B, self.g = B, torch.Generator().manual_seed(5)
        pool = [torch.full((LAYERS, n_pages, PAGE, KV, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        zeros = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
        self.cache = B.sol_attn3d_paged_cache(pool[0], pool[1], zeros(n_streams, width) - 1, zeros(n_streams), zeros(n_pages))
        self.gain = [(1.0 + 0.1 * torch.randn(D, generator=self.g)) for _ in range(2)]
        # what every stream holds, per layer, in fp64: rotated keys as the cache has them (bf16), values
        self.k = [[torch.zeros(0, KV, D, dtype=torch.float64) for _ in range(n_streams)] for _ in range(LAYERS)]
        self.v = [[torch.zeros(0, KV, D, dtype=torch.float64) for _ in range(n_streams)] for _ in range(LAYERS)]
        states = torch.randn(100, 2, KV, D, generator=self.g).bfloat16()
        self.prompt, dev = states, states.cuda()
        self.ctx_begin, self.ctx_len = [0, 40, 40, 0], [40, 60, 60, 40]
        self.ctx_kv = dev

    def status(self, n):
        return torch.full((n,), -1, dtype=torch.int32, device="cuda")

    def chunk(self, seqs, streams, pos0, causal):
        """Appends a chunk to each of the streams and attends, in every layer."""
        B = self.B
        sizes = [s[0] + s[1] * s[2] * s[3] for s in seqs]
        st, n, status = ints(streams), sum(sizes), self.status(len(streams))
        B.sol_attn3d_cache_reserve(self.cache, st, ints(sizes), status)
        attn = B.Attn3d(seqs, HEADS, D, rope(D), q_strides=((HEADS + 2 * KV) * D, D))
        heads_plan = B.Attn3d(seqs, HEADS, D, rope(D))
        ctx = B.sol_attn3d_context(self.ctx_kv[:, 0], self.ctx_kv[:, 1], ints([self.ctx_begin[s] for s in streams]), ints([self.ctx_len[s] for s in streams]), 60)
        ws = torch.empty(max(B.sol_attn3d_paged_workspace_bytes(heads_plan.plan, self.cache), B.sol_attn3d_cross_workspace_bytes(heads_plan.plan, ctx)),
                         dtype=torch.uint8, device="cuda")
        for layer in range(LAYERS):
            x = torch.randn(n, HEADS + 2 * KV, D, generator=self.g).bfloat16()
            dx = x.cuda()
            q, out, cross = (torch.empty(n, HEADS, D, dtype=torch.bfloat16, device="cuda") for _ in range(3))
            B.sol_attn3d_cache_append(attn.plan, dx[:, :HEADS], dx[:, HEADS:HEADS + KV], dx[:, HEADS + KV:], q, self.cache, layer, streams=st, pos0=ints(pos0),
                                      q_gain=self.gain[0].cuda(), k_gain=self.gain[1].cuda(), eps=EPS)
            B.sol_attn3d_forward_paged(heads_plan.plan, q, self.cache, layer, out, streams=st, causal_block=causal, workspace=ws)
            B.sol_attn3d_forward_cross(heads_plan.plan, q, ctx, cross, workspace=ws)
            torch.cuda.synchronize()
            assert heads_plan.status() == 0 and status.tolist() == [0] * len(streams)
            at = 0
            for seq, s, m, off in zip(seqs, streams, sizes, pos0):
                rows = x[at:at + m]
                k = so.rotate_chunk(so.normalise(rows[:, HEADS:HEADS + KV], self.gain[1], EPS), seq, rope(D), 10000.0, off)
                # the cache's own rounding of K is taken from the cache: what attention has to match is attention over it
                table, held = self.cache.table[s].tolist(), self.k[layer][s].shape[0]
                got = torch.stack([self.cache.k[layer, table[j // PAGE], j % PAGE] for j in range(held, held + m)]).cpu().double()
                assert bool(((got - k).abs() <= torch.finfo(torch.bfloat16).eps / 2 * 1.01 * k.abs() + 1e-5).all())
                self.k[layer][s] = torch.cat([self.k[layer][s], got])
                self.v[layer][s] = torch.cat([self.v[layer][s], rows[:, HEADS + KV:].double()])
                total = held + m
                ref, mag = so.attend(q[at:at + m].cpu(), self.k[layer][s], self.v[layer][s], so.key_limits(m, total, causal))
                close(out[at:at + m].cpu(), ref, mag)
                p = self.prompt[self.ctx_begin[s]:self.ctx_begin[s] + self.ctx_len[s]]
                ref, mag = so.attend(q[at:at + m].cpu(), p[:, 0], p[:, 1], so.key_limits(m, len(p), 0))
                close(cross[at:at + m].cpu(), ref, mag)
                at += m

    def steps(self, streams):
        """One more token of each stream with the single-token forms."""
        B = self.B
        n, st, status = len(streams), ints(streams), self.status(len(streams))
        B.sol_attn3d_cache_reserve(self.cache, st, ints([1] * n), status)
        attn = B.Attn3d([(0, 1, 1, 1)] * n, HEADS, D, rope(D))
        ws = torch.empty(B.sol_attn3d_paged_step_workspace_bytes(self.cache, n, HEADS), dtype=torch.uint8, device="cuda")
        for layer in range(LAYERS):
            q, k, v = (torch.randn(n, h, D, generator=self.g).bfloat16() for h in (HEADS, KV, KV))
            rot, out = torch.empty(n, HEADS, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, HEADS, D, dtype=torch.bfloat16, device="cuda")
            pos = [[self.k[layer][s].shape[0], 3, 4] for s in streams]
            B.sol_attn3d_cache_append(attn.plan, q.cuda(), k.cuda(), v.cuda(), rot, self.cache, layer, streams=st, pos0=ints(pos))
            B.sol_attn3d_paged_step(rot, self.cache, layer, out, streams=st, workspace=ws)
            torch.cuda.synchronize()
            assert status.tolist() == [0] * n
            for i, s in enumerate(streams):
                ref_k = so.rotate_chunk(k[i:i + 1], (0, 1, 1, 1), rope(D), 10000.0, pos[i])
                self.k[layer][s] = torch.cat([self.k[layer][s], ref_k.bfloat16().double()])
                self.v[layer][s] = torch.cat([self.v[layer][s], v[i:i + 1].double()])
                ref, mag = so.attend(rot[i:i + 1].cpu(), self.k[layer][s], self.v[layer][s], so.key_limits(1, self.k[layer][s].shape[0], 0))
                close(out[i:i + 1].cpu(), ref, mag, slack=2e-3)           # (a key in half a dozen thousand rounds the other way: 2^-8 of one score)

    def fork(self, parents, streams):
        status = self.status(len(streams))
        ws = torch.empty(self.B.sol_attn3d_cache_workspace_bytes(self.cache, len(streams)), dtype=torch.uint8, device="cuda")
        self.B.sol_attn3d_cache_fork(self.cache, ints(parents), ints(streams), status, ws)
        assert status.tolist() == [0] * len(streams)
        for layer in range(LAYERS):
            for p, s in zip(parents, streams):
                self.k[layer][s], self.v[layer][s] = self.k[layer][p].clone(), self.v[layer][p].clone()

    def window(self, streams, sink, last):
        keep = torch.zeros(len(streams), 24 * PAGE, dtype=torch.uint8)
        for i, s in enumerate(streams):
            n = self.k[0][s].shape[0]
            keep[i, :sink] = 1
            keep[i, max(0, n - last):n] = 1
        status = self.status(len(streams))
        ws = torch.empty(self.B.sol_attn3d_cache_workspace_bytes(self.cache, len(streams)), dtype=torch.uint8, device="cuda")
        self.B.sol_attn3d_cache_compact(self.cache, ints(streams), keep.cuda(), status, ws)
        assert status.tolist() == [0] * len(streams)
        for layer in range(LAYERS):
            for i, s in enumerate(streams):
                on = keep[i, :self.k[layer][s].shape[0]].bool()
                self.k[layer][s], self.v[layer][s] = self.k[layer][s][on], self.v[layer][s][on]

    def free(self, streams):
        self.B.sol_attn3d_cache_free(self.cache, ints(streams))
        for layer in range(LAYERS):
            for s in streams:
                self.k[layer][s], self.v[layer][s] = self.k[layer][s][:0], self.v[layer][s][:0]


def test_streams_grow_branch_and_forget():
    loop = Loop()
    loop.chunk([(5, 2, 3, 7), (0, 1, 3, 7)], [0, 1], [[0, 0, 0], [9, 2, 1]], 21)
    loop.chunk([(0, 3, 3, 7), (0, 1, 3, 7)], [1, 0], [[10, 2, 1], [2, 0, 0]], 0)
    loop.fork([0, 1], [2, 3])
    loop.chunk([(0, 1, 3, 7), (0, 2, 3, 7), (0, 1, 3, 7)], [2, 0, 3], [[3, 0, 0], [3, 0, 0], [13, 2, 1]], 21)
    loop.window([0, 3], 5, 40)
    loop.chunk([(0, 1, 3, 7)] * 4, [3, 1, 0, 2], [[14, 2, 1], [13, 2, 1], [5, 0, 0], [4, 0, 0]], 1)
    loop.steps([2, 0, 3])
    loop.free([1, 2])
    loop.fork([3], [1])
    loop.window([1], 0, 3)
    loop.steps([1, 3, 0])
    loop.free([0, 1, 3])
    assert int(loop.cache.refs.abs().sum()) == 0 and int(loop.cache.lens.sum()) == 0
