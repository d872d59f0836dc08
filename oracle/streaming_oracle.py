"""fp64 CPU oracle of streaming generation: attention of new tokens over cached or encoded keys, the pass that fills a paged cache,
and the bookkeeping of its pages.  TEST INFRASTRUCTURE ONLY.

Plain definitions, nothing tiled, nothing rounded; imports nothing from the package.
    out = softmax(q k^T / sqrt(d)) v over the keys that count; query head h uses K/V head h // (heads // kv_heads); no key: zeros
    new token i of n, in a stream of N: keys below N, or with blocks of B new tokens below N - n + (i // B + 1) * B
    k~ = rotate(k / sqrt(mean(k^2) + eps) * gain, position + offset)
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import torch

from .attn3d_oracle import F64, layout_positions, rope_rotate, widen


def key_limits(n_new: int, n_all: int, block: int) -> torch.Tensor:
    """Keys below limit[i] count for new token i."""
    if block == 0:
        return torch.full((n_new,), n_all)
    i = torch.arange(n_new)
    return (n_all - n_new + (i // block + 1) * block).clamp(0, n_all)


def attend(q, k, v, limits: torch.Tensor, valid: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """q [n, heads, d], k, v [N, kv_heads, d], limits [n], valid bool [N] or None -> (out, sum of p |v|), both [n, heads, d].
    Keys that count for no row take no part, whatever they hold."""
    q = widen(q)
    n, heads, d = q.shape
    out, mag = torch.zeros(n, heads, d, dtype=F64), torch.zeros(n, heads, d, dtype=F64)
    keep = torch.arange(k.shape[0]) < (int(limits.max()) if n else 0)
    if valid is not None:
        keep = keep & valid
    at = keep.nonzero()[:, 0]
    if len(at) == 0:
        return out, mag
    k, v = widen(k[at]), widen(v[at])
    seen = at[None] < limits[:, None]                                   # [n, keys]
    rows = seen.any(1)
    for h in range(heads):
        kv = h // (heads // k.shape[1])
        s = (q[rows, h] @ k[:, kv].T) / d ** 0.5
        s = s.masked_fill(~seen[rows], -float("inf"))
        e = torch.exp(s - s.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
        out[rows, h], mag[rows, h] = p @ v[:, kv], p @ v[:, kv].abs()
    return out, mag


def normalise(x, gain, eps: float) -> torch.Tensor:
    x = widen(x)
    return x if gain is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * widen(gain)


def rotate_chunk(x, seq, rope_dims, theta: float, pos0=(0, 0, 0)) -> torch.Tensor:
    """One chunk [n, heads, d] (prefix, then grid), positions of the grid offset by pos0."""
    _, pos, has = layout_positions([seq])
    return rope_rotate(widen(x), pos, has, rope_dims, theta, origin=pos0)


OK, BAD_STREAM, NO_ROOM, NO_PAGES, NOT_EMPTY = range(5)


class PageBook:
    """Streams and pages as plain lists.  `rows` maps every (page, row) to what it holds; the calls move its entries."""

    def __init__(self, table: Sequence[Sequence[int]], lens: Sequence[int], refs: Sequence[int], page: int, rows=None):
        self.table, self.lens, self.refs, self.page = [list(r) for r in table], list(lens), list(refs), page
        self.rows = rows if rows is not None else {(p, r): (p, r) for p in range(len(refs)) for r in range(page)}

    def pages(self, tokens: int) -> int:
        return -(-tokens // self.page)

    def _named(self, streams: Sequence[int], i: int) -> bool:
        return 0 <= streams[i] < len(self.lens) and streams[i] not in streams[:i]

    def _admit(self, needs: List[Optional[int]]) -> List[bool]:
        """Requests that need pages are served until the first one for which the free pages do not suffice."""
        left, open_, served = self.refs.count(0), True, []
        for need in needs:
            if need is None or need == 0:
                served.append(need is not None)
                continue
            open_ = open_ and need <= left
            left -= need if open_ else 0
            served.append(open_)
        return served

    def _take(self) -> int:
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def reserve(self, streams, amount):
        status, needs = [], []
        for i, (s, a) in enumerate(zip(streams, amount)):
            needs.append(None)
            if not self._named(streams, i) or a < 0:
                status.append(BAD_STREAM)
            elif self.lens[s] + a > len(self.table[s]) * self.page:
                status.append(NO_ROOM)
            else:
                status.append(OK)
                needs[-1] = self.pages(self.lens[s] + a) - self.pages(self.lens[s])
        for i, ok in enumerate(self._admit(needs)):
            if ok:
                s = streams[i]
                for c in range(self.pages(self.lens[s]), self.pages(self.lens[s] + amount[i])):
                    self.table[s][c] = self._take()
                self.lens[s] += amount[i]
            elif status[i] == OK:
                status[i] = NO_PAGES
        return status

    def fork(self, parents, streams):
        status, needs, was = [], [], [r[:] for r in self.table]
        n = list(self.lens)
        for i, (p, s) in enumerate(zip(parents, streams)):
            needs.append(None)
            if not self._named(streams, i) or not 0 <= p < len(n):
                status.append(BAD_STREAM)
            elif n[s] != 0:
                status.append(NOT_EMPTY)
            else:
                status.append(OK)
                needs[-1] = 1 if n[p] % self.page else 0
        for i, ok in enumerate(self._admit(needs)):
            if not ok:
                status[i] = status[i] or NO_PAGES
                continue
            p, s = parents[i], streams[i]
            full, rest = divmod(n[p], self.page)
            for c in range(full):
                self.table[s][c] = was[p][c]
                self.refs[was[p][c]] += 1
            if rest:
                new = self.table[s][full] = self._take()
                for r in range(rest):
                    self.rows[new, r] = self.rows[was[p][full], r]
            self.lens[s] = n[p]
        return status

    def compact(self, streams, keep):
        status, needs, plan = [], [], []
        refs = list(self.refs)
        for i, s in enumerate(streams):
            needs.append(None)
            plan.append(None)
            if not self._named(streams, i):
                status.append(BAD_STREAM)
                continue
            status.append(OK)
            kept = [j for j in range(self.lens[s]) if j < len(keep[i]) and keep[i][j]]
            first = next((a for a, j in enumerate(kept) if a != j), len(kept))
            begin = first // self.page
            if first == len(kept) and (first % self.page == 0 or refs[self.table[s][begin]] <= 1):
                begin = self.pages(first)
            needs[-1], plan[-1] = max(0, self.pages(len(kept)) - begin), (kept, begin)
        gone, rows = [], dict(self.rows)
        for i, ok in enumerate(self._admit(needs)):
            if not ok:
                status[i] = status[i] or NO_PAGES
                continue
            s, (kept, begin) = streams[i], plan[i]
            old = self.table[s][:self.pages(self.lens[s])]
            gone += old[begin:]
            for c in range(begin, len(old)):
                self.table[s][c] = -1
            for c in range(begin, self.pages(len(kept))):
                new = self.table[s][c] = self._take()
                for r, j in enumerate(kept[c * self.page:(c + 1) * self.page]):
                    self.rows[new, r] = rows[old[j // self.page], j % self.page]
            self.lens[s] = len(kept)
        for p in gone:
            self.refs[p] -= 1
        return status

    def free(self, streams):
        status = []
        for i, s in enumerate(streams):
            if not self._named(streams, i):
                status.append(BAD_STREAM)
                continue
            status.append(OK)
            for c in range(self.pages(self.lens[s])):
                self.refs[self.table[s][c]] -= 1
                self.table[s][c] = -1
            self.lens[s] = 0
        return status
