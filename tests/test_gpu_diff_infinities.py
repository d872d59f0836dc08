"""Infinities in q, k and v where they count: both forms of the differential attention give what the formula gives."""
import math

import pytest
import torch

from oracle import diff_linear_oracle as dlo
from test_gpu_diff import TOL, make

pytestmark = pytest.mark.gpu

N, HEADS = 150, 4


def cases():
    inf = math.inf
    return {
        "one key": [("k", (5, 0, 3), inf)],
        "one key, second map, late tile": [("k", (140, 1, 7), -inf)],
        "one query": [("q", (7, 1, 0), -inf)],
        "one value": [("v", (9, 0, 4), inf)],
        "one value of the second head": [("v", (149, 3, 63), -inf)],
        "every key of a map": [("k", (slice(None), 0, 0), -inf)],
        "NaN in a key": [("k", (30, 2, 1), math.nan)],
    }


def oracle(q, k, v, o):
    refs, mags = [], []
    for pair in range(HEADS // 2):
        h = slice(2 * pair, 2 * pair + 2)
        qq, kk, vv = dlo.widen(q[:, h]), dlo.widen(k[:, h]), dlo.widen(v[:, h]).reshape(-1, 128)
        refs.append(dlo.diff_rows(qq, kk, vv, o["lam"], None)[0])
        mags.append(dlo.diff_rows(qq, kk, vv.abs(), -abs(o["lam"]), None)[0])
    return torch.stack(refs, 1).reshape(-1, HEADS, 64), torch.stack(mags, 1).reshape(-1, HEADS, 64)


def compare(got, ref, mag):
    """Not finite in the same places, and where it is an infinity the same one; elsewhere within 4 times the contract's relative
    error of the two maps' magnitudes (as for single rows in the other tests)."""
    got = got.double().cpu()
    assert torch.equal(got.isnan(), ref.isnan())
    ok = torch.isfinite(ref)
    assert torch.equal(got[~ok & ~ref.isnan()], ref[~ok & ~ref.isnan()])
    assert bool(((got - ref).abs()[ok] <= 4 * TOL * mag[ok]).all())


@pytest.mark.parametrize("name", list(cases()))
def test_over_a_plan(name):
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, o = make([(N, 0, 1, 1)], HEADS, 310, gain=False)     # prefix tokens: not rotated
    for which, at, value in cases()[name]:
        dict(q=q, k=k, v=v)[which][at] = value
    if name == "every key of a map":
        q[:, 0, 0] = q[:, 0, 0].abs() + 0.5
    out = torch.full_like(q, 7.0)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
    torch.cuda.synchronize()
    assert attn.status() == 0
    compare(out, *oracle(q, k, v, o))
    attn.close()


def test_rotated_infinities_and_large_finite_values():
    """Rotation of an infinity gives infinities or NaN in its pair of dims; rows whose scores do not see them stay finite, and
    finite magnitudes above 65504 saturate."""
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, _ = make([(0, 2, 5, 7)], 2, 311, gain=False)
    q[3, 0, 2] = math.inf
    q[4, 1, 9] = 3e38
    out = torch.full_like(q, 7.0)
    B.sol_attn3d_forward_diff(attn.plan, q, k, v, out, None, w)
    torch.cuda.synchronize()
    rows = out.reshape(70, -1).isnan().all(1)
    assert bool(rows[3]) and int(rows.sum()) == 1 and int(out.isnan().any(-1).any(-1).sum()) == 1
    attn.close()


@pytest.mark.parametrize("capacity", [N, 8192])                              # one CTA per row and pair, and several
@pytest.mark.parametrize("name", list(cases()))
def test_step(name, capacity):
    from paper_2609_35110_b200 import binding as B
    attn, (q, k, v), w, o = make([(N, 0, 1, 1)], HEADS, 312, gain=False)
    attn.close()
    for which, at, value in cases()[name]:
        dict(q=q, k=k, v=v)[which][at] = value
    if name == "every key of a map":
        q[:, 0, 0] = q[:, 0, 0].abs() + 0.5
    cache = [torch.full((1, capacity, HEADS, 64), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for c, x in zip(cache, (k, v)):
        c[0, :N] = x
    rows = [0, 7, 60, 149]
    b = len(rows)
    ws = torch.empty(B.sol_attn3d_diff_step_workspace_bytes(b, HEADS, 64, capacity), dtype=torch.uint8, device="cuda")
    lens = torch.full((b,), N, dtype=torch.int32, device="cuda")
    slots = torch.zeros(b, dtype=torch.int32, device="cuda")
    for mask in (None, torch.ones(1, capacity, dtype=torch.uint8, device="cuda")):
        out = torch.full((b, HEADS, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        B.sol_attn3d_diff_step(q[rows].contiguous(), *cache, lens, out, w, ws, key_mask=mask, slots=slots)
        torch.cuda.synchronize()
        ref, mag = oracle(q, k, v, o)
        compare(out, ref[rows], mag[rows])
