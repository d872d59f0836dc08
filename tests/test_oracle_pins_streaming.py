"""Pins of the streaming oracle: closed forms, brute force, and what the bookkeeping must keep whatever is called."""
import itertools
import math
import random

import torch

from oracle import attn3d_oracle as orc
from oracle import streaming_oracle as so


def test_limits():
    assert so.key_limits(3, 10, 0).tolist() == [10, 10, 10]
    assert so.key_limits(3, 10, 1).tolist() == [8, 9, 10]
    assert so.key_limits(5, 12, 2).tolist() == [9, 9, 11, 11, 12]
    assert so.key_limits(4, 2, 1).tolist() == [0, 0, 1, 2]


def test_attend_by_hand():
    g = torch.Generator().manual_seed(0)
    q, k, v = torch.randn(3, 4, 8, generator=g), torch.randn(6, 2, 8, generator=g), torch.randn(6, 2, 8, generator=g)
    valid = torch.tensor([1, 0, 1, 1, 1, 0]).bool()
    out, mag = so.attend(q, k, v, torch.tensor([0, 3, 6]), valid)
    assert bool((out[0] == 0).all()) and bool((mag[0] == 0).all())
    for i, keys in ((1, [0, 2]), (2, [0, 2, 3, 4])):
        for h in range(4):
            w = [math.exp(sum(float(q[i, h, d]) * float(k[j, h // 2, d]) for d in range(8)) / math.sqrt(8)) for j in keys]
            for d in range(8):
                want = sum(x * float(v[j, h // 2, d]) for x, j in zip(w, keys)) / sum(w)
                assert abs(float(out[i, h, d]) - want) < 1e-12
    # what does not count may be anything; one key alone is its value
    k2, v2 = k.clone(), v.clone()
    k2[~valid], v2[~valid] = float("nan"), float("inf")
    assert torch.equal(so.attend(q, k2, v2, torch.tensor([0, 3, 6]), valid)[0], out)
    one, _ = so.attend(q, k, v, torch.full((3,), 6), torch.arange(6) == 4)
    assert torch.equal(one, v[4].double().repeat_interleave(2, 0).expand(3, 4, 8))


def test_attend_is_the_dense_oracle_without_a_past():
    g = torch.Generator().manual_seed(1)
    seq, d = (3, 2, 3, 4), 64
    q, k, v = (torch.randn(27, 2, d, generator=g).bfloat16() for _ in range(3))
    ref = orc.attn3d_oracle(q, k, v, [seq], (16, 24, 24), 10000.0)
    rot = lambda x: so.rotate_chunk(x, seq, (16, 24, 24), 10000.0)
    out, _ = so.attend(rot(q), rot(k), v, so.key_limits(27, 27, 0))
    assert torch.allclose(out, ref, rtol=0, atol=1e-12)


def test_offsets_continue_a_grid():
    """Frames of a clip, appended one at a time at their place, have the keys of the whole clip."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4 * 6, 3, 64, generator=g)
    whole = so.rotate_chunk(x, (0, 4, 2, 3), (16, 24, 24), 10000.0)
    parts = [so.rotate_chunk(x[6 * t:6 * t + 6], (0, 1, 2, 3), (16, 24, 24), 10000.0, (t, 0, 0)) for t in range(4)]
    assert torch.allclose(torch.cat(parts), whole, rtol=0, atol=1e-12)


def check(book, contents):
    """Counts agree with the tables, nobody writes what another one reads, and every stream holds what it should."""
    held = [row[:book.pages(n)] for row, n in zip(book.table, book.lens)]
    for p in range(len(book.refs)):
        assert book.refs[p] == sum(row.count(p) for row in held)
    for row, n in zip(held, book.lens):
        if n % book.page:
            assert book.refs[row[-1]] == 1                              # a partly filled page has one holder
    for row, n, want in zip(held, book.lens, contents):
        assert [book.rows[row[j // book.page], j % book.page] for j in range(n)] == want


def test_bookkeeping_keeps_its_promises():
    rng, fresh = random.Random(3), itertools.count()
    for _ in range(30):
        page, streams, width, pages = rng.choice([2, 3, 5]), rng.randint(2, 6), rng.randint(1, 5), rng.randint(1, 25)
        book = so.PageBook([[-1] * width for _ in range(streams)], [0] * streams, [0] * pages, page)
        contents = [[] for _ in range(streams)]
        for _ in range(25):
            who = [rng.randint(-1, streams) for _ in range(rng.randint(1, 4))]
            what = rng.choice(["reserve", "reserve", "fork", "compact", "free"])
            if what == "reserve":
                amount = [rng.randint(0, 2 * page) for _ in who]
                for s, a, st in zip(who, amount, book.reserve(who, amount)):
                    for _ in range(a if st == so.OK else 0):            # the new tokens are written, each with something of its own
                        j = len(contents[s])
                        book.rows[book.table[s][j // page], j % page] = mark = next(fresh)
                        contents[s].append(mark)
            elif what == "fork":
                parents, was = [rng.randint(-1, streams) for _ in who], [c[:] for c in contents]
                for s, p, st in zip(who, parents, book.fork(parents, who)):
                    if st == so.OK:
                        contents[s] = was[p][:]
            elif what == "compact":
                keep = [[rng.random() < 0.7 for _ in range(rng.randint(1, width * page))] for _ in who]
                for s, k, st in zip(who, keep, book.compact(who, keep)):
                    if st == so.OK:
                        contents[s] = [x for j, x in enumerate(contents[s]) if j < len(k) and k[j]]
            else:
                for s, st in zip(who, book.free(who)):
                    if st == so.OK:
                        contents[s] = []
            check(book, contents)
