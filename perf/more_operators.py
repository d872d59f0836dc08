"""Cases of the operators of streaming generation: attention of new tokens over a paged K/V cache (a chunk of frames, or one
token per stream), the pass that brings new tokens into that cache (norm, rotation, write), the opening, growing, thinning and
closing of streams in it, and cross attention to an encoder's states.

``own`` false: plain form, elementary torch operations in fp32, rounded once at the end.  ``own`` true: the calls a
program makes of the framework.

Tensors are bf16.  A cache holds pages of `page` tokens, [layers, pages, page, kv_heads, head_dim]; a stream's token j is row
j % page of page table[stream, j // page].  Query head h uses K/V head h // (heads // kv_heads).
    paged:   row i of a chunk of n new tokens, the last n of a stream of N:  out = softmax(q k^T / sqrt(D)) v  over the valid keys
             below N, or with causal = B > 0 below N - n + (i // B + 1) * B.
    append:  k~ = rotate(k / sqrt(mean(k^2) + eps) * gain), the same for q; adjacent pairs of dims, axes (t, h, w), positions offset
             per stream, prefix tokens not rotated.
    pages:   fork shares the full pages and copies the last, partly filled one; compact keeps chosen tokens, the pages before the
             first dropped one stay, the others are written anew; new pages are the free ones of the lowest index.
    cross:   out = softmax(q k^T / sqrt(D)) v  over the valid states of the sequence's context.
"""
import math

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # three latent frames of the low-resolution stage against the stage's whole length: one block of a streaming generator
        {"name": "paged_lowres", "op": "paged", "seqs": "0x3x30x52", "lens": "25216", "heads": 40, "kv_heads": 40, "head_dim": 128, "page": 64, "causal": 0, "mask": False},
        # four streams at different places, shared K/V heads, every frame sees the frames up to its own, evicted keys masked
        {"name": "paged_frames", "op": "paged", "seqs": "77x2x15x26,0x3x15x26,0x1x15x26,512x0x1x1", "lens": "857,4144,12700,512", "heads": 48, "kv_heads": 8, "head_dim": 128, "page": 48,
         "causal": 390, "mask": True},
        # few new rows, a long past: the keys have to be split
        {"name": "paged_long", "op": "paged", "seqs": "0x1x6x10", "lens": "111856", "heads": 40, "kv_heads": 8, "head_dim": 128, "page": 128, "causal": 1, "mask": False},
        # one token of one stream, short past: latency
        {"name": "step_short", "op": "step", "batch": 1, "heads": 8, "kv_heads": 8, "head_dim": 64, "page": 16, "shortest": 333, "longest": 333, "mask": False},
        # a batch of streams of different length
        {"name": "step_batch", "op": "step", "batch": 24, "heads": 40, "kv_heads": 8, "head_dim": 128, "page": 64, "shortest": 77, "longest": 12736, "mask": True},
        # the tokens of one decoding step of a batch: latency
        {"name": "append_step", "op": "append", "seqs": ",".join(["0x1x1x1"] * 16), "lens": ",".join(str(100 + 17 * i) for i in range(16)), "heads": 40, "kv_heads": 8, "head_dim": 128, "page": 16,
         "norm": True},
        # the new frames of the low-resolution stage, one block
        {"name": "append_lowres", "op": "append", "seqs": "0x3x30x52", "lens": "9360", "heads": 40, "kv_heads": 40, "head_dim": 128, "page": 64, "norm": True},
        # a branch of every stream (guidance, candidates), each with room for its next frame, all layers of a small stack
        {"name": "pages_fork", "op": "pages", "what": "fork", "streams": 12, "shortest": 77, "longest": 4144, "layers": 8, "kv_heads": 8, "head_dim": 128, "page": 128, "grow": 390},
        # prompt and latest frames stay, what lies between goes
        {"name": "pages_window", "op": "pages", "what": "compact", "streams": 4, "shortest": 3000, "longest": 12736, "layers": 8, "kv_heads": 8, "head_dim": 128, "page": 64, "sink": 256, "window": 3120},
        # one token per stream against its prompt
        {"name": "cross_step", "op": "cross", "single": 24, "seqs": "", "ctx": ",".join(str(77 + 18 * i) for i in range(24)), "heads": 40, "kv_heads": 40, "head_dim": 128, "mask": False},
        # low-resolution stage, prompt states of an encoder
        {"name": "cross_lowres", "op": "cross", "single": 0, "seqs": "256x16x30x52", "ctx": "512", "heads": 40, "kv_heads": 40, "head_dim": 128, "mask": False},
        # four packed videos of different size, padded prompts, one without a prompt
        {"name": "cross_packed", "op": "cross", "single": 0, "seqs": "256x8x30x52,256x4x7x13,0x16x30x52,77x1x6x10", "ctx": "512,77,0,1025", "heads": 48, "kv_heads": 48, "head_dim": 64, "mask": True},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _grid(rng, tokens):
    """A sequence of about `tokens` tokens: prefix and grid."""
    text = min(rng.choice([0, 0, 1, 77, 256, 511]), tokens // 2)
    left = max(1, tokens - text)
    t = rng.randint(1, max(1, min(16, left)))
    h = max(1, min(45, int(math.sqrt(left / t * rng.uniform(0.3, 0.9)))))
    w = max(1, left // (t * h))
    return (text, t, h, w)


def _text(seqs):
    return ",".join("x".join(map(str, s)) for s in seqs)


def _size(seq):
    return seq[0] + seq[1] * seq[2] * seq[3]


def draw(rng):
    op = rng.choice(["paged", "paged", "step", "append", "pages", "cross", "cross"])
    head_dim = rng.choice([64, 128])
    kv_heads, group = rng.choice([(1, 1), (2, 1), (5, 1), (12, 1), (40, 1), (1, 6), (2, 3), (4, 2), (5, 4), (8, 5), (8, 6), (2, 16), (1, 40)])
    heads = kv_heads * group
    shape = {"heads": heads, "kv_heads": kv_heads, "head_dim": head_dim}
    page = rng.choice([16, 32, 48, 64, 80, 128, 256])
    if op == "paged":
        seqs = [_grid(rng, _log_uniform(rng, 1, 4000)) for _ in range(rng.randint(1, 5))]
        lens = [_size(s) + rng.choice([0, 1, _log_uniform(rng, 1, 20000)]) for s in seqs]
        causal = rng.choice([0, 0, 1, rng.randint(2, 400)])
        return {"op": op, "seqs": _text(seqs), "lens": ",".join(map(str, lens)), **shape, "page": page, "causal": causal, "mask": rng.random() < 0.3}
    if op == "step":
        batch = _log_uniform(rng, 1, 64)
        longest = _log_uniform(rng, 1, min(60000, 2400000 // (batch * kv_heads)))
        return {"op": op, "batch": batch, **shape, "page": page, "shortest": rng.randint(0, longest), "longest": longest, "mask": rng.random() < 0.4}
    if op == "append":
        seqs = [_grid(rng, _log_uniform(rng, 1, 3000)) for _ in range(rng.randint(1, 5))]
        lens = [_size(s) + rng.randint(0, 3000) for s in seqs]
        return {"op": op, "seqs": _text(seqs), "lens": ",".join(map(str, lens)), **shape, "page": page, "norm": rng.random() < 0.7}
    if op == "pages":
        streams, longest = rng.randint(1, 12), _log_uniform(rng, 16, 4144)
        case = {"op": op, "what": rng.choice(["fork", "compact"]), "streams": streams, "shortest": rng.randint(1, longest), "longest": longest, "layers": rng.randint(1, 8),
                "kv_heads": min(8, kv_heads), "head_dim": head_dim, "page": page}
        if case["what"] == "fork":
            return {**case, "grow": rng.randint(0, 400)}
        return {**case, "sink": rng.randint(0, longest // 2), "window": rng.randint(0, longest)}
    if rng.random() < 0.3:
        batch = rng.randint(1, 48)
        return {"op": "cross", "single": batch, "seqs": "", "ctx": ",".join(str(rng.randint(0, 600)) for _ in range(batch)), **shape, "mask": rng.random() < 0.4}
    seqs = [_grid(rng, _log_uniform(rng, 1, 8000)) for _ in range(rng.randint(1, 4))]
    ctx = [rng.choice([0, 1, 77, 256, 512, rng.randint(1, 1500)]) for _ in seqs]
    return {"op": "cross", "single": 0, "seqs": _text(seqs), "ctx": ",".join(map(str, ctx)), **shape, "mask": rng.random() < 0.4}


def _seqs(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["seqs"].split(",")]


def _numbers(text):
    return [int(x) for x in text.split(",")]


def _offsets(sizes):
    cu = [0]
    for n in sizes:
        cu.append(cu[-1] + n)
    return cu


def _spread(case, n):
    """n lengths from the shortest to the longest."""
    low, high = case["shortest"], case["longest"]
    return [high if n == 1 else low + (high - low) * i // (n - 1) for i in range(n)]


def _rope_dims(head_dim):
    return (16, 24, 24) if head_dim == 64 else (32, 48, 48)


def _pages_of(n, page):
    return -(-n // page)


def _kept(case, n):
    """Which of a stream's n tokens stay: the first `sink` and the last `window`."""
    return [j for j in range(n) if j < case["sink"] or j >= n - case["window"]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, D = case["op"], case["head_dim"]

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        x = torch.empty(shape, dtype=dtype, device="cuda")
        flat = x.view(-1)
        for a in range(0, flat.numel(), 1 << 27):
            m = min(1 << 27, flat.numel() - a)
            flat[a:a + m] = torch.randn(m, generator=gen, device="cuda") * scale
        return x

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def shuffled(n):
        return torch.randperm(n, generator=gen, device="cuda").to(torch.int32)

    def pool(lens, layers, spare, width):
        """A cache whose streams hold lens[i] tokens in pages from all over the pool; what no stream holds is garbage, too."""
        page, counts = case["page"], [_pages_of(n, case["page"]) for n in lens]
        n_pages = sum(counts) + spare
        s["k"], s["v"] = (normal(layers, n_pages, page, case["kv_heads"], D) for _ in range(2))
        ids, table, at = shuffled(n_pages), torch.full((len(lens), max(1, width)), -1, dtype=torch.int32, device="cuda"), 0
        s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        for i, c in enumerate(counts):
            table[i, :c] = ids[at:at + c]
            at += c
        s["refs"][ids[:at].long()] = 1
        s["table"], s["lens"], s["lens_host"] = table, ints(lens), list(lens)

    s = {"case": case}
    if op in ("paged", "append"):
        seqs = _seqs(case)
        s["seqs"], s["cu"] = seqs, _offsets([_size(x) for x in seqs])
        n, lens = s["cu"][-1], _numbers(case["lens"])
        order = shuffled(len(seqs)).tolist()                         # sequence i is stream order[i]
        by_stream = [0] * len(seqs)
        for i, st in enumerate(order):
            by_stream[st] = lens[i]
        pool(by_stream, 1, 3, _pages_of(max(lens), case["page"]))
        s["streams"], s["streams_host"] = ints(order), order
        if op == "paged":
            s["q"] = normal(n, case["heads"], D)
            s["out"] = torch.zeros_like(s["q"])
            s["mask"] = (torch.rand(len(seqs), max(lens), generator=gen, device="cuda") < 0.9).to(torch.uint8) if case["mask"] else None
        else:
            heads, kv = case["heads"], case["kv_heads"]
            qkv = normal(n, heads + 2 * kv, D, scale=1.5)            # one packed projection output
            s["q"], s["k_new"], s["v_new"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
            s["q_out"] = torch.zeros(n, heads, D, dtype=torch.bfloat16, device="cuda")
            s["gains"] = [1.0 + normal(D, scale=0.1, dtype=torch.float32) for _ in range(2)] if case["norm"] else [None, None]
            s["pos0"] = torch.randint(0, 200, (len(seqs), 3), generator=gen, device="cuda", dtype=torch.int32)
    elif op == "step":
        b = case["batch"]
        lens = _spread(case, b)
        pool(lens, 1, 3, _pages_of(max(lens), case["page"]))
        s["streams"] = shuffled(b)
        s["streams_host"] = s["streams"].tolist()
        s["q"] = normal(b, case["heads"], D)
        s["out"] = torch.zeros_like(s["q"])
        s["mask"] = (torch.rand(b, max(1, max(lens)), generator=gen, device="cuda") < 0.9).to(torch.uint8) if case["mask"] else None
    elif op == "pages":
        n = case["streams"]
        lens = _spread(case, n)
        grow = case.get("grow", 0)
        spare = sum(_pages_of(x + grow, case["page"]) + 1 for x in lens)
        pool(lens + [0] * n, case["layers"], spare, _pages_of(max(lens) + grow, case["page"]))
        s["parents"], s["branches"] = ints(list(range(n))), ints(list(range(n, 2 * n)))
        s["grow"] = ints([grow] * n)
        s["status"] = torch.full((3, n), -1, dtype=torch.int32, device="cuda")
        if case["what"] == "compact":
            keep = torch.zeros(n, max(1, max(lens)), dtype=torch.uint8)
            for i, x in enumerate(lens):
                keep[i, _kept(case, x)] = 1
            s["keep"] = keep.cuda()
    else:
        lens = _numbers(case["ctx"])
        cu = _offsets(lens)
        s["begins"], s["lens"], s["ctx"] = ints(cu[:-1]), ints(lens), list(zip(cu, lens))
        kv = normal(max(1, cu[-1]), 2 * case["kv_heads"], D)         # one packed projection output
        s["k"], s["v"] = kv[:, :case["kv_heads"]], kv[:, case["kv_heads"]:]
        s["mask"] = None
        if case["mask"]:                                             # the second half of every context is padding, the last one's whole
            m = torch.ones(max(1, cu[-1]), dtype=torch.uint8)
            for a, n in s["ctx"]:
                m[a + (n + 1) // 2:a + n] = 0
            if len(lens) > 1:
                m[cu[-2]:] = 0
            s["mask"] = m.cuda()
        seqs = [(1, 0, 1, 1)] * case["single"] if case["single"] else _seqs(case)
        s["cu"] = _offsets([_size(x) for x in seqs])
        s["q"] = normal(s["cu"][-1], case["heads"], D)
        s["out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2609_35110_b200 import binding as B

        def scratch(nbytes):
            return torch.empty(nbytes, dtype=torch.uint8, device="cuda")

        if op == "cross":
            s["context"] = B.sol_attn3d_context(s["k"], s["v"], s["begins"], s["lens"], max(lens), key_mask=s["mask"])
            if case["single"]:
                s["ws"] = scratch(B.sol_attn3d_cross_step_workspace_bytes(s["context"], case["single"], case["heads"]))
            else:
                s["attn"] = B.Attn3d(seqs, case["heads"], D, _rope_dims(D))
                s["ws"] = scratch(B.sol_attn3d_cross_workspace_bytes(s["attn"].plan, s["context"]))
        else:
            s["cache"] = B.sol_attn3d_paged_cache(s["k"], s["v"], s["table"], s["lens"], s["refs"])
            if op in ("paged", "append"):
                st = (s["q"].stride(0), D)
                s["attn"] = B.Attn3d(seqs, case["heads"], D, _rope_dims(D), q_strides=st)
            if op == "paged":
                s["ws"] = scratch(B.sol_attn3d_paged_workspace_bytes(s["attn"].plan, s["cache"]))
            if op == "step":
                s["ws"] = scratch(B.sol_attn3d_paged_step_workspace_bytes(s["cache"], case["batch"], case["heads"]))
            if op == "pages":
                s["ws"] = scratch(B.sol_attn3d_cache_workspace_bytes(s["cache"], case["streams"]))
    return s


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"paged": _plain_paged, "step": _plain_step, "append": _plain_append, "pages": _plain_pages, "cross": _plain_cross}[op](s)
    from paper_2609_35110_b200 import binding as B
    if op == "paged":
        B.sol_attn3d_forward_paged(s["attn"].plan, s["q"], s["cache"], 0, s["out"], streams=s["streams"], key_mask=s["mask"], causal_block=s["case"]["causal"], workspace=s["ws"])
        return s["out"]
    if op == "step":
        B.sol_attn3d_paged_step(s["q"], s["cache"], 0, s["out"], streams=s["streams"], key_mask=s["mask"], workspace=s["ws"])
        return s["out"]
    if op == "append":
        B.sol_attn3d_cache_append(s["attn"].plan, s["q"], s["k_new"], s["v_new"], s["q_out"], s["cache"], 0, streams=s["streams"], pos0=s["pos0"],
                                  q_gain=s["gains"][0], k_gain=s["gains"][1], eps=EPS)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if op == "cross":
        if s["case"]["single"]:
            B.sol_attn3d_cross_step(s["q"], s["context"], s["out"], workspace=s["ws"])
        else:
            B.sol_attn3d_forward_cross(s["attn"].plan, s["q"], s["context"], s["out"], workspace=s["ws"])
        return s["out"]
    # the branches of the last pass are closed, new ones opened
    B.sol_attn3d_cache_free(s["cache"], s["branches"], s["status"][0])
    B.sol_attn3d_cache_fork(s["cache"], s["parents"], s["branches"], s["status"][1], s["ws"])
    if s["case"]["what"] == "fork":
        B.sol_attn3d_cache_reserve(s["cache"], s["branches"], s["grow"], s["status"][2])
    else:
        B.sol_attn3d_cache_compact(s["cache"], s["branches"], s["keep"], s["status"][2], s["ws"])
    return {x: s[x] for x in ("table", "refs", "lens", "status", "k", "v")}


# ------------------------------------------------------------------------------------------------ plain forms
def _attend(q, k, v, valid):
    """q [rows, heads, D], k, v [keys, kv_heads, D], valid [rows or 1, keys] -> bf16 [rows, heads, D]; a row without keys is zeros."""
    n, heads, D = q.shape
    group = heads // k.shape[1]
    out = torch.zeros_like(q)
    if k.shape[0] == 0 or n == 0:
        return out
    k, v = k.float().permute(1, 2, 0), v.float().permute(1, 0, 2)                       # [kv, D, keys], [kv, keys, D]
    step = max(1, (1 << 30) // (heads * k.shape[2]))
    for a in range(0, n, step):
        b = min(a + step, n)
        x = q[a:b].float().view(b - a, -1, group, D).permute(1, 2, 0, 3).flatten(1, 2)  # [kv, group * rows, D]
        z = (x @ k).mul_(D ** -0.5).view(x.shape[0], group, b - a, -1)
        if valid is not None:
            z = z.masked_fill_(~(valid if valid.shape[0] == 1 else valid[a:b]), -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
        z = z / z.sum(-1, keepdim=True).clamp(min=1e-38)
        out[a:b] = (z.flatten(1, 2) @ v).view(-1, group, b - a, D).permute(2, 0, 1, 3).reshape(b - a, heads, D).bfloat16()
    return out


def _gather(s, stream, n):
    """K and V rows of a stream's first n tokens."""
    page = s["case"]["page"]
    j = torch.arange(n, device="cuda")
    row = s["table"][stream, j // page].long() * page + j % page
    return (s[x][0].flatten(0, 1)[row] for x in ("k", "v"))


def _plain_paged(s):
    out, causal = torch.empty_like(s["out"]), s["case"]["causal"]
    for a, b, st in zip(s["cu"], s["cu"][1:], s["streams_host"]):
        n = s["lens_host"][st]
        k, v = _gather(s, st, n)
        j, valid = torch.arange(n, device="cuda"), None
        if causal:
            valid = j < (n - (b - a) + (torch.arange(b - a, device="cuda") // causal + 1) * causal)[:, None]
        if s["mask"] is not None:
            m = s["mask"][st, :n].bool()[None]
            valid = m if valid is None else valid & m
        out[a:b] = _attend(s["q"][a:b], k, v, valid)
    return out


def _plain_step(s):
    out = torch.empty_like(s["out"])
    for i, st in enumerate(s["streams_host"]):
        n = s["lens_host"][st]
        k, v = _gather(s, st, n)
        out[i:i + 1] = _attend(s["q"][i:i + 1], k, v, None if s["mask"] is None else s["mask"][st, None, :n].bool())
    return out


def _plain_cross(s):
    out = torch.empty_like(s["out"])
    for a, b, (c, n) in zip(s["cu"], s["cu"][1:], s["ctx"]):
        out[a:b] = _attend(s["q"][a:b], s["k"][c:c + n], s["v"][c:c + n], None if s["mask"] is None else s["mask"][None, c:c + n].bool())
    return out


def _plain_append(s):
    case = s["case"]
    D, page = case["head_dim"], case["page"]

    def norm(x, gain):
        x = x.float()
        return x if gain is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain

    k, v = s["k"][0].flatten(0, 1), s["v"][0].flatten(0, 1)
    for i, (a, b, st, (text, T, H, W)) in enumerate(zip(s["cu"], s["cu"][1:], s["streams_host"], s["seqs"])):
        p = torch.arange(T * H * W, device="cuda")
        angles = []
        for axis, (x, d) in enumerate(zip((p // max(1, H * W), p // W % H, p % W), _rope_dims(D))):
            omega = 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
            angles.append((x + s["pos0"][i, axis])[:, None].double() * omega)
        angles = torch.cat(angles, 1)[:, None]
        c, sn = angles.cos().float(), angles.sin().float()

        def rotate(x):
            even, odd, r = x[text:, :, 0::2], x[text:, :, 1::2], 2 * c.shape[-1]
            even, odd, rest = even[..., :r // 2], odd[..., :r // 2], x[text:, :, r:]
            turned = torch.stack([even * c - odd * sn, even * sn + odd * c], -1).flatten(-2)
            return torch.cat([x[:text], torch.cat([turned, rest], -1)])

        s["q_out"][a:b] = rotate(norm(s["q"][a:b], s["gains"][0])).bfloat16()
        j = torch.arange(b - a, device="cuda") + s["lens_host"][st] - (b - a)
        row = s["table"][st, j // page].long() * page + j % page
        k[row] = rotate(norm(s["k_new"][a:b], s["gains"][1])).bfloat16()
        v[row] = s["v_new"][a:b]
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_pages(s):
    case = s["case"]
    page, table, refs, lens = case["page"], s["table"], s["refs"], s["lens"]
    src, dst = s["parents"].long(), s["branches"].long()
    col = torch.arange(table.shape[1], device="cuda")

    def count(streams, rows, by):
        """refs += by for the chosen entries of the streams' table rows"""
        refs.index_add_(0, table[streams].clamp(min=0).flatten().long(), (rows * by).to(torch.int32).flatten())

    def take(need):
        """need[i] free pages for request i, lowest index first: [requests, columns] page ids, valid for column < need[i]"""
        free = torch.sort((refs != 0).to(torch.int32), stable=True).indices
        at = (torch.cumsum(need, 0) - need)[:, None] + col
        return free[at.clamp(max=len(free) - 1)].to(torch.int32)

    # close the branches
    held = col < ((lens[dst] + page - 1) // page)[:, None]
    count(dst, held, -1)
    table[dst] = torch.where(held, -1, table[dst])
    lens[dst] = 0
    # open them again
    n = lens[src].long()
    full, part = n // page, n % page
    new = take((part > 0).long())[:, 0]
    count(src, col < full[:, None], 1)
    refs[new[part > 0].long()] = 1
    last = (col == full[:, None]) & (part > 0)[:, None]
    table[dst] = torch.where(col < full[:, None], table[src], torch.where(last, new[:, None], table[dst]))
    lens[dst] = n.to(torch.int32)
    for i in range(len(src)):
        old, fresh = table[src[i]].gather(0, full[i:i + 1].clamp(max=len(col) - 1)).long(), new[i:i + 1].long()
        rows = (torch.arange(page, device="cuda") < part[i])[None, None, :, None, None]
        for x in ("k", "v"):
            s[x][:, fresh] = torch.where(rows, s[x][:, old], s[x][:, fresh])
    s["status"].zero_()
    if case["what"] == "fork":
        before = (lens[dst].long() + page - 1) // page
        lens[dst] += s["grow"]
        need = (lens[dst].long() + page - 1) // page - before
        new, k = take(need), col - before[:, None]
        fill = (k >= 0) & (k < need[:, None])
        table[dst] = torch.where(fill, new.gather(1, k.clamp(min=0)), table[dst])
        count(dst, fill, 1)
    else:
        pos = torch.arange(s["keep"].shape[1], device="cuda")
        there = pos < lens[dst].long()[:, None]
        kept = there & s["keep"].bool()
        n_old, n_new = lens[dst].long(), kept.sum(1)
        first = torch.where(there & ~kept, pos, n_old[:, None]).amin(1)                 # the first dropped token
        shared = refs[table[dst].clamp(min=0).long()].gather(1, (first // page).clamp(max=len(col) - 1)[:, None])[:, 0] > 1
        stays = (n_new == first) & ((first % page == 0) | ~shared)                      # a prefix stays: nothing moves
        begin = torch.where(stays, (n_new + page - 1) // page, first // page)           # pages before this one stay
        need = (n_new + page - 1) // page - begin
        need = need.clamp(min=0)
        new, k, old = take(need), col - begin[:, None], table[dst]
        fill = (k >= 0) & (k < need[:, None])
        gone = (k >= 0) & (col < ((n_old + page - 1) // page)[:, None])
        fresh = torch.where(fill, new.gather(1, k.clamp(min=0)), torch.where(gone, -1, old))
        for i in range(len(dst)):
            at = kept[i].nonzero()[:, 0]
            j = torch.arange(len(at), device="cuda")
            at, j = at[j >= begin[i] * page], j[j >= begin[i] * page]
            a, b = (t.long()[x // page] * page + x % page for t, x in ((old[i], at), (fresh[i], j)))
            for x in ("k", "v"):
                s[x].flatten(1, 2)[:, b] = s[x].flatten(1, 2)[:, a]
        count(dst, gone, -1)
        table[dst] = fresh
        count(dst, fill, 1)
        lens[dst] = n_new.to(torch.int32)
    return {x: s[x] for x in ("table", "refs", "lens", "status", "k", "v")}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, D, kv = case["op"], case["head_dim"], case["kv_heads"]
    row = kv * D * 2                                                                     # bytes of one token's K, or V
    if op == "paged":
        bytes_, flops = 0, 0
        for n, N in zip((_size(x) for x in _seqs(case)), _numbers(case["lens"])):
            B = case["causal"]
            pairs = n * N if not B else sum(min(N, N - n + (i // B + 1) * B) for i in range(n))
            share = 0.9 if case["mask"] else 1.0
            bytes_ += 2 * n * case["heads"] * D * 2 + share * N * 2 * row + (N if case["mask"] else 0)
            flops += share * 4 * pairs * D * case["heads"]
        return {"bytes": bytes_, "flops": flops}
    if op == "step":
        tokens, share = sum(_spread(case, case["batch"])), 0.9 if case["mask"] else 1.0
        return {"bytes": tokens * (share * 2 * row + (1 if case["mask"] else 0)) + 2 * case["batch"] * case["heads"] * D * 2, "flops": share * 4 * tokens * D * case["heads"]}
    if op == "append":
        n = sum(_size(x) for x in _seqs(case))
        return {"bytes": 2 * n * (case["heads"] + 2 * kv) * D * 2, "flops": 8 * n * (case["heads"] + kv) * D}
    if op == "pages":
        page, moved = case["page"], 0
        for n in _spread(case, case["streams"]):
            moved += n % page
            if case["what"] == "compact":
                kept = _kept(case, n)
                first = next((i for i, j in enumerate(kept) if i != j), len(kept))
                moved += 0 if len(kept) == first and first % page == 0 else max(0, len(kept) - first // page * page)
        return {"bytes": 2 * moved * 2 * row * case["layers"], "flops": 0}
    rows = [1] * case["single"] if case["single"] else [_size(x) for x in _seqs(case)]
    ctx = _numbers(case["ctx"])
    if case["mask"]:
        ctx = [(n + 1) // 2 for n in ctx[:-1]] + [ctx[-1] if len(ctx) == 1 else 0]
    return {"bytes": sum(2 * a * case["heads"] * D * 2 + n * 2 * row for a, n in zip(rows, ctx)), "flops": sum(4 * a * n for a, n in zip(rows, ctx)) * D * case["heads"]}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, D, f = case["op"], case["head_dim"], torch.float64
    if op in ("paged", "step", "cross"):
        out = torch.zeros(s["out"].shape, dtype=f, device="cuda")
        group = case["heads"] // case["kv_heads"]
        table = s["table"].tolist() if op != "cross" else None
        for i, (a, b) in enumerate(zip(s["cu"], s["cu"][1:]) if op != "step" else ((i, i + 1) for i in range(case["batch"]))):
            if op == "cross":
                begin, n = s["ctx"][i]
                k, v = s["k"][begin:begin + n], s["v"][begin:begin + n]
                seen = None if s["mask"] is None else s["mask"][begin:begin + n] != 0
            else:
                stream = s["streams_host"][i]
                n = s["lens_host"][stream]
                pages = table[stream][:_pages_of(n, case["page"])]
                k, v = (torch.cat([s[x][0, p] for p in pages])[:n] if pages else s[x][0, 0, :0] for x in ("k", "v"))
                seen = None if s["mask"] is None else s["mask"][stream, :n] != 0
            seen = torch.ones(n, dtype=torch.bool, device="cuda") if seen is None else seen
            before = seen.new_zeros(b - a, 0)
            if op == "paged" and case["causal"]:
                frame = torch.div(torch.arange(b - a, device="cuda"), case["causal"], rounding_mode="floor")
                before = torch.arange(n, device="cuda")[None] - (n - (b - a)) < ((frame + 1) * case["causal"])[:, None]
            for h in range(case["heads"]):
                kh, vh = k[:, h // group].to(f)[seen], v[:, h // group].to(f)[seen]
                for r in range(a, b, 8192):
                    e = min(b, r + 8192)
                    z = s["q"][r:e, h].to(f) @ kh.T / math.sqrt(D)
                    if before.shape[1]:
                        z[~before[r - a:e - a][:, seen]] = -math.inf
                    if z.shape[1]:
                        out[r:e, h] = torch.nan_to_num(torch.softmax(z, 1)) @ vh         # (rows whose limit leaves nothing: zeros)
        return out
    if op == "append":
        res = {"q": s["q"].to(f), "k": s["k"].to(f), "v": s["v"].to(f)}
        page = case["page"]
        for i, (text, T, H, W) in enumerate(s["seqs"]):
            a, b, stream = s["cu"][i], s["cu"][i + 1], s["streams_host"][i]
            turn = torch.ones(b - a, D // 2, dtype=torch.complex128, device="cuda")
            grid = torch.cartesian_prod(*(torch.arange(x, dtype=f, device="cuda") for x in (T, H, W))).view(-1, 3) + s["pos0"][i].to(f)
            at = 0
            for axis, width in enumerate(_rope_dims(D)):
                for j in range(width // 2):
                    angle = grid[:, axis] / 10000.0 ** (2.0 * j / width)
                    turn[text:, at] = torch.polar(torch.ones_like(angle), angle)
                    at += 1

            def whole(x, gain):
                x = x.to(f)
                if gain is not None:
                    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.to(f)
                return torch.view_as_real(torch.view_as_complex(x.reshape(b - a, -1, D // 2, 2)) * turn[:, None]).flatten(-2)

            k, v = whole(s["k_new"][a:b], s["gains"][1]), s["v_new"][a:b].to(f)
            res["q"][a:b] = whole(s["q"][a:b], s["gains"][0])
            start, row = s["lens_host"][stream] - (b - a), s["table"][stream].tolist()
            done = 0
            while done < b - a:                                      # page by page
                p, r = divmod(start + done, page)
                m = min(page - r, b - a - done)
                res["k"][0, row[p], r:r + m], res["v"][0, row[p], r:r + m] = k[done:done + m], v[done:done + m]
                done += m
        return res
    # pages: the bookkeeping in lists
    table, refs, lens = s["table"].tolist(), s["refs"].tolist(), list(s["lens_host"])
    res = {"status": torch.zeros_like(s["status"]), "k": s["k"].to(f), "v": s["v"].to(f)}
    page, n = case["page"], case["streams"]

    def fresh():
        p = refs.index(0)
        refs[p] = 1
        return p

    for i in range(n):
        whole, rest = divmod(lens[i], page)
        for c in range(whole):
            table[n + i][c] = table[i][c]
            refs[table[i][c]] += 1
        if rest:
            p = table[n + i][whole] = fresh()
            for x in ("k", "v"):
                res[x][:, p, :rest] = res[x][:, table[i][whole], :rest]
        lens[n + i] = lens[i]
    if case["what"] == "fork":
        for i in range(n, 2 * n):
            for c in range(_pages_of(lens[i], page), _pages_of(lens[i] + case["grow"], page)):
                table[i][c] = fresh()
            lens[i] += case["grow"]
    else:
        released = []
        source = {x: res[x].clone() for x in ("k", "v")}
        for i in range(n, 2 * n):
            kept = _kept(case, lens[i])
            first = next((a for a, b in enumerate(kept) if a != b), len(kept))
            pages = table[i][:_pages_of(lens[i], page)]
            if len(kept) == first and (first % page == 0 or refs[pages[first // page]] == 1):
                begin = _pages_of(first, page)
            else:
                begin = first // page
            for c in range(begin, len(pages)):
                released.append(pages[c])
                table[i][c] = -1
            for c in range(begin, _pages_of(len(kept), page)):
                p = table[i][c] = fresh()
                at = kept[c * page:(c + 1) * page]
                src = torch.tensor([pages[a // page] * page + a % page for a in at], device="cuda")
                for x in ("k", "v"):
                    res[x][:, p, :len(at)] = source[x].flatten(1, 2)[:, src]
            lens[i] = len(kept)
        for p in released:
            refs[p] -= 1
    for x, t in (("table", table), ("refs", refs), ("lens", lens)):
        res[x] = torch.tensor(t, dtype=torch.int32, device="cuda")
    return {x: res[x] for x in ("table", "refs", "lens", "status", "k", "v")}
