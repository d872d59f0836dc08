"""Streaming entry points take q and out by the plan's strides; a tensor that has others is refused instead of being read wrongly."""
import pytest
import torch

from paper_2609_35110_b200 import binding as B
from paper_2609_35110_b200 import build as build_mod

D = 64


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build_mod.build_library()


@pytest.mark.parametrize("heads", [1, 3])
def test_tensors_and_plans(heads):
    row = heads * D
    dense = B.sol_attn3d_plan(1, heads, D, 1, 2, 5, 0, (16, 24, 24))
    packed = B.sol_attn3d_plan_ex([(0, 1, 2, 5)], heads, D, (16, 24, 24), 10000.0, q_strides=(row + 2 * D, D), out_strides=(0, 0))
    major = B.sol_attn3d_plan_ex([(0, 1, 2, 5)], heads, D, (16, 24, 24), 10000.0, out_strides=(D, 10 * D))
    x = torch.zeros(10, heads + 2, D, dtype=torch.bfloat16)
    part, whole, by_head = x[:, :heads], x[:, :heads].contiguous(), torch.zeros(heads, 10, D, dtype=torch.bfloat16).transpose(0, 1)
    wide = torch.zeros(10, heads, 2 * D, dtype=torch.bfloat16)[..., ::2]
    check = lambda plan, name, t: B._check_strides(plan, name, t, heads, D)
    for plan, name, t in ((dense, "q", whole), (dense, "out", whole), (packed, "q", part), (packed, "out", whole), (major, "out", by_head), (major, "q", whole.view(10, row)),
                          (packed, "q", x.view(10, row + 2 * D)[:, :row]), (dense, "q", part[:1]), (dense, "q", x), (dense, "out", x.view(-1))):
        check(plan, name, t)
    for plan, name, t in ((dense, "q", part), (dense, "out", part), (packed, "q", whole), (packed, "out", part), (dense, "q", wide),
                          (dense, "q", x.view(10, row + 2 * D)[:, :row]), (packed, "q", whole.view(10, row))):
        with pytest.raises(ValueError, match="strides"):
            check(plan, name, t)
    if heads > 1:
        for plan, name, t in ((dense, "q", by_head), (major, "out", whole), (major, "out", whole.view(10, row))):
            with pytest.raises(ValueError, match="strides"):
                check(plan, name, t)
    for p in (dense, packed, major):
        B.sol_attn3d_destroy(p)


@pytest.mark.gpu
def test_entry_points():
    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    attn = B.Attn3d([(0, 1, 2, 5)], 3, D, (16, 24, 24))
    x = torch.zeros(10, 5, D, dtype=torch.bfloat16, device="cuda")
    part, whole = x[:, :3], torch.zeros(10, 3, D, dtype=torch.bfloat16, device="cuda")
    pool = [torch.zeros(1, 4, 16, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = B.sol_attn3d_paged_cache(pool[0], pool[1], ints([[0, 1]]), ints([10]))
    ctx = B.sol_attn3d_context(x[:, 3:4], x[:, 4:], ints([0]), ints([10]), 10)
    kv = x[:, 3:4]
    for call in (lambda: B.sol_attn3d_forward_paged(attn.plan, part, cache, 0, whole), lambda: B.sol_attn3d_forward_paged(attn.plan, whole, cache, 0, part),
                 lambda: B.sol_attn3d_forward_cross(attn.plan, part, ctx, whole), lambda: B.sol_attn3d_forward_cross(attn.plan, whole, ctx, part),
                 lambda: B.sol_attn3d_cache_append(attn.plan, part, kv, kv, torch.empty_like(whole), cache, 0)):
        with pytest.raises(ValueError, match="strides"):
            call()
    B.sol_attn3d_cache_append(attn.plan, whole, kv, kv, torch.empty_like(whole), cache, 0)
    torch.cuda.synchronize()
