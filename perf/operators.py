"""Cases of the attention operators beside the dense softmax attention: differential attention (over the tokens of a
plan, and for one new token over a cache) and linear attention with a decay per head (over the tokens of a plan, and
one token at a time).

``own`` false: plain form, elementary torch operations in fp32, rounded once at the end.  ``own`` true: the calls a
program makes of the framework.

Tensors are bf16 unless said otherwise.  Differential attention pairs the heads 2i and 2i+1 (head_dim 64): two softmax
maps over one value tensor of 128 dims (the two heads' V side by side),
    x = softmax(q1 k1^T / 8) v - lambda * softmax(q2 k2^T / 8) v,
    lambda = exp(lq1 . lk1) - exp(lq2 . lk2) + lambda_init,
    out = (1 - lambda_init) * x / sqrt(mean(x^2) + eps) * gain          (without a gain: out = x).
Linear attention keeps one fp32 state S [head_dim, head_dim] per sequence and head:
    S_t = exp(log_decay) * S_{t-1} + k_t^T v_t,      out_t = scale * q_t S_t;      a masked key adds nothing to S.
"""
import math

import torch

own = False

LOWRES = (256, 16, 30, 52)        # text tokens, T, H, W of the low-resolution stage
HIGHRES = (256, 31, 45, 80)       # high-resolution stage
EPS = 1e-5


def listed():
    return [
        # the correctness grid: 256 tokens; all latency
        {"name": "diff_tiny", "op": "diff", "seqs": "0x4x8x8", "heads": 4, "layer": 0, "gain": True, "mask": False, "refs": 0.0},
        # classifier-free-guidance pair, prompts of 512 and 77 tokens padded to 512, a mid-size grid with a ragged tail
        {"name": "diff_cfg_pair", "op": "diff", "seqs": "512x8x15x26,512x8x15x26", "heads": 16, "layer": 3, "gain": True, "mask": True, "refs": 0.0},
        # low-resolution stage, one block's attention
        {"name": "diff_lowres", "op": "diff", "seqs": "256x16x30x52", "heads": 40, "layer": 11, "gain": True, "mask": False, "refs": 0.0},
        # reference tokens (60 % of the video) are keys only; without the norm
        {"name": "diff_refs", "op": "diff", "seqs": "256x8x30x52", "heads": 48, "layer": 7, "gain": False, "mask": False, "refs": 0.6},
        # one new token, short cache: latency
        {"name": "diff_step_short", "op": "diff_step", "batch": 1, "heads": 8, "capacity": 512, "shortest": 333, "longest": 333, "gain": True, "mask": False},
        # a batch of streams of different length, in shuffled slots of the cache
        {"name": "diff_step_batch", "op": "diff_step", "batch": 24, "heads": 40, "capacity": 12736, "shortest": 77, "longest": 12736, "gain": True, "mask": True},
        # one stream at the length of the high-resolution stage
        {"name": "diff_step_highres", "op": "diff_step", "batch": 1, "heads": 40, "capacity": 111856, "shortest": 111856, "longest": 111856, "gain": True, "mask": False},
        # the correctness grid
        {"name": "linear_tiny", "op": "linear", "seqs": "0x4x8x8", "heads": 4, "head_dim": 64, "mask": False, "carry": True},
        # four packed videos of different size, one prompt padded, no carried state
        {"name": "linear_packed", "op": "linear", "seqs": "256x8x30x52,256x4x7x13,256x16x30x52,77x1x6x10", "heads": 48, "head_dim": 64, "mask": True, "carry": False},
        # high-resolution stage, continued from the state of an earlier clip
        {"name": "linear_highres", "op": "linear", "seqs": "256x31x45x80", "heads": 40, "head_dim": 128, "mask": False, "carry": True},
        # one token of one stream
        {"name": "linear_step_one", "op": "linear_step", "batch": 1, "heads": 40, "head_dim": 128, "slots": 1, "idle": 0},
        # many streams, some rows of the batch idle
        {"name": "linear_step_batch", "op": "linear_step", "batch": 96, "heads": 48, "head_dim": 128, "slots": 112, "idle": 5},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _grid(rng, tokens):
    """A sequence of about `tokens` tokens: prefix and grid."""
    text = min(rng.choice([0, 0, 1, 77, 256, 511]), tokens // 2)
    left = max(1, tokens - text)
    t = rng.randint(1, max(1, min(31, left)))
    h = max(1, min(45, int(math.sqrt(left / t * rng.uniform(0.3, 0.9)))))
    w = max(1, left // (t * h))
    return (text, t, h, w)


def draw(rng):
    op = rng.choice(["diff", "diff_step", "linear", "linear_step"])
    if op in ("diff", "linear"):
        head_dim = 64 if op == "diff" else rng.choice([64, 128])
        heads = 2 * rng.randint(1, 20) if op == "diff" else rng.randint(1, 48)
        total = _log_uniform(rng, 1, 20000 if op == "diff" else 80000)
        n = rng.randint(1, 4)
        seqs = [_grid(rng, max(1, int(total * rng.uniform(0.1, 1.0) / n))) for _ in range(n)]
        case = {"op": op, "seqs": ",".join("x".join(map(str, s)) for s in seqs), "heads": heads, "mask": rng.random() < 0.4}
        if op == "diff":
            return {**case, "layer": rng.randint(0, 40), "gain": rng.random() < 0.7, "refs": rng.choice([0.0, 0.0, 0.3, 0.8])}
        return {**case, "head_dim": head_dim, "carry": rng.random() < 0.5}
    if op == "diff_step":
        batch, heads = _log_uniform(rng, 1, 48), 2 * rng.randint(1, 20)
        longest = _log_uniform(rng, 1, min(110000, 11000000 // (batch * heads)))
        return {"op": op, "batch": batch, "heads": heads, "capacity": longest + rng.randint(0, 64), "shortest": rng.randint(0, longest), "longest": longest,
                "gain": rng.random() < 0.7, "mask": rng.random() < 0.4}
    batch = _log_uniform(rng, 1, 96)
    return {"op": op, "batch": batch, "heads": rng.randint(1, 48), "head_dim": rng.choice([64, 128]), "slots": batch + rng.randint(0, 16), "idle": rng.randint(0, batch // 4)}


def _seqs(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["seqs"].split(",")]


def _offsets(seqs):
    cu = [0]
    for text, t, h, w in seqs:
        cu.append(cu[-1] + text + t * h * w)
    return cu


def _rope_dims(head_dim):
    return (16, 24, 24) if head_dim == 64 else (32, 48, 48)


def _key_mask(seqs, on):
    """A quarter of the first sequence's prompt is valid, all but the last token of the others' (padding)."""
    if not on:
        return None
    cu = _offsets(seqs)
    m = torch.ones(cu[-1], dtype=torch.uint8)
    for s, (text, *_rest) in enumerate(seqs):
        m[cu[s] + (text // 4 if s == 0 else max(0, text - 1)): cu[s] + text] = 0
    return m.cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        x = torch.empty(shape, dtype=dtype, device="cuda")
        rows = max(1, (1 << 27) // max(1, x.numel() // max(1, shape[0])))
        for a in range(0, shape[0], rows):
            x[a:a + rows] = torch.randn((min(rows, shape[0] - a),) + tuple(shape[1:]), generator=gen, device="cuda") * scale
        return x

    s = {"case": case}
    heads = case["heads"]
    if case["op"] in ("diff", "diff_step"):
        layer = case.get("layer", 5)
        s["lams"] = [normal(64, scale=0.1, dtype=torch.float32) for _ in range(4)]
        s["lambda_init"] = 0.8 - 0.6 * math.exp(-0.3 * layer)
        s["gain"] = 1.0 + normal(128, scale=0.1, dtype=torch.float32) if case["gain"] else None
    if case["op"] in ("diff", "linear"):
        seqs = _seqs(case)
        D = case.get("head_dim", 64)
        n = _offsets(seqs)[-1]
        qkv = normal(n, 3 * heads * D).view(n, 3, heads, D)          # one packed projection output
        if case["op"] == "linear":
            qkv[:, 1] *= D ** -0.5
        s["q"], s["k"], s["v"] = qkv[:, 0], qkv[:, 1], qkv[:, 2]
        s["mask"] = _key_mask(seqs, case["mask"])
        s["out"] = torch.zeros(n, heads, D, dtype=torch.bfloat16, device="cuda")
        if case["op"] == "diff":
            want = torch.ones(n, dtype=torch.uint8)
            for a, (text, t, h, w) in zip(_offsets(seqs), seqs):
                want[a + text: a + text + int(case["refs"] * t * h * w)] = 0
            s["want"] = want.cuda() if case["refs"] else None
        else:
            # decays from 1 - 2^-2 to 1 - 2^-12 over the heads
            e = torch.linspace(2, 12, heads, dtype=torch.float64)
            s["log_decay"] = torch.log1p(-(2.0 ** -e)).float().cuda()
            s["scale"] = 1.0
            s["state_in"] = normal(len(seqs), heads, D, D, dtype=torch.float32) if case["carry"] else None
            s["state_out"] = torch.zeros(len(seqs), heads, D, D, dtype=torch.float32, device="cuda")
    elif case["op"] == "diff_step":
        b, cap = case["batch"], case["capacity"]
        s["q"] = normal(b, heads, 64)
        s["k"], s["v"] = normal(b, cap, heads, 64), normal(b, cap, heads, 64)
        lens = torch.randint(case["shortest"], case["longest"] + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
        lens[0] = case["longest"]
        s["lens"] = lens
        s["slots"] = torch.randperm(b, generator=gen, device="cuda").to(torch.int32)
        s["mask"] = (torch.rand(b, cap, generator=gen, device="cuda") < 0.9).to(torch.uint8) if case["mask"] else None
        s["out"] = torch.zeros(b, heads, 64, dtype=torch.bfloat16, device="cuda")
    else:
        b, D = case["batch"], case["head_dim"]
        s["q"], s["k"], s["v"] = normal(b, heads, D), normal(b, heads, D, scale=D ** -0.5), normal(b, heads, D)
        e = torch.linspace(2, 12, heads, dtype=torch.float64)
        s["log_decay"] = torch.log1p(-(2.0 ** -e)).float().cuda()
        s["scale"] = 1.0
        s["state_in"] = normal(case["slots"], heads, D, D, dtype=torch.float32)
        s["state_out"] = s["state_in"].clone()                       # slots that no row names keep what they hold
        slots = torch.randperm(case["slots"], generator=gen, device="cuda")[:b].to(torch.int32)
        if case["idle"]:
            slots[:case["idle"]] = -1
        s["slots"] = slots
        s["out"] = torch.zeros(b, heads, D, dtype=torch.bfloat16, device="cuda")
    if own:
        from paper_2609_35110_b200 import binding as B
        if case["op"] in ("diff", "diff_step"):
            s["weights"] = B.sol_attn3d_diff_weights(*s["lams"], s["lambda_init"], s["gain"], EPS)
        if case["op"] in ("diff", "linear"):
            st = (3 * heads * D, D)
            s["attn"] = B.Attn3d(seqs, heads, D, _rope_dims(D), q_strides=st, k_strides=st, v_strides=st)
        if case["op"] == "linear":
            s["scratch"] = torch.empty(B.sol_attn3d_linear_workspace_bytes(s["attn"].plan), dtype=torch.uint8, device="cuda")
        if case["op"] == "diff_step":
            s["scratch"] = torch.empty(B.sol_attn3d_diff_step_workspace_bytes(b, heads, 64, cap), dtype=torch.uint8, device="cuda")
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2609_35110_b200 import binding as B
        s = state
        if op == "diff":
            B.sol_attn3d_forward_diff(s["attn"].plan, s["q"], s["k"], s["v"], s["out"], s["mask"], s["weights"], s["want"])
            return s["out"]
        if op == "diff_step":
            B.sol_attn3d_diff_step(s["q"], s["k"], s["v"], s["lens"], s["out"], s["weights"], s["scratch"], key_mask=s["mask"], slots=s["slots"])
            return s["out"]
        if op == "linear":
            B.sol_attn3d_forward_linear(s["attn"].plan, s["q"], s["k"], s["v"], s["out"], s["mask"], s["log_decay"], s["scale"],
                                        s["state_in"], s["state_out"], s["scratch"])
        else:
            B.sol_attn3d_linear_step(s["q"], s["k"], s["v"], s["out"], s["log_decay"], s["scale"], s["state_in"], s["state_out"], slots=s["slots"])
        return {"out": s["out"], "state": s["state_out"]}
    return {"diff": _plain_diff, "diff_step": _plain_diff_step, "linear": _plain_linear, "linear_step": _plain_linear_step}[op](state)


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_rotate(x, seq):
    """[n, heads, 64] -> fp32, the video tokens rotated by their (t, h, w); angles in fp64."""
    text, T, H, W = seq
    x = x.float()
    if T * H * W == 0:
        return x
    pos = torch.arange(T * H * W, device=x.device)
    angles = []
    for p, d in zip((pos // (H * W), pos // W % H, pos % W), _rope_dims(x.shape[-1])):
        omega = 10000.0 ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
        angles.append(p[:, None].double() * omega)
    a = torch.cat(angles, 1)[:, None]
    c, s = a.cos().float(), a.sin().float()
    even, odd = x[text:, :, 0::2], x[text:, :, 1::2]
    return torch.cat([x[:text], torch.stack([even * c - odd * s, even * s + odd * c], -1).flatten(-2)])


def _plain_lambda(s):
    a, b, c, d = s["lams"]
    return torch.exp((a * b).sum()) - torch.exp((c * d).sum()) + s["lambda_init"]


def _plain_norm(s, x):
    if s["gain"] is None:
        return x
    return (1.0 - s["lambda_init"]) * x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * s["gain"]


def _softmax(z, valid):
    if valid is None:
        p = torch.exp(z - z.amax(-1, keepdim=True))
        return p / p.sum(-1, keepdim=True)
    z = z.masked_fill(~valid, -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
    return p / p.sum(-1, keepdim=True).clamp(min=1e-38)


def _plain_diff(s):
    seqs, heads = _seqs(s["case"]), s["case"]["heads"]
    cu, lam = _offsets(seqs), _plain_lambda(s)
    out = s["out"].clone()
    for a, b, seq in zip(cu, cu[1:], seqs):
        n = b - a
        q, k = (_plain_rotate(s[x][a:b], seq).view(n, heads // 2, 2, 64).permute(2, 1, 0, 3) for x in ("q", "k"))      # [2, pairs, n, 64]
        v = s["v"][a:b].float().reshape(n, heads // 2, 128).permute(1, 0, 2)
        valid = None if s["mask"] is None else s["mask"][a:b].bool()
        rows = torch.arange(n, device=q.device) if s["want"] is None else s["want"][a:b].nonzero()[:, 0]
        step = max(1, (1 << 31) // (heads * n))                      # rows at a time, so that the scores fit
        for r in rows.split(step):
            p = _softmax(q[:, :, r] @ k.transpose(-1, -2) * 0.125, valid)
            x = _plain_norm(s, (p[0] - lam * p[1]) @ v)
            out[a + r] = x.permute(1, 0, 2).reshape(len(r), heads, 64).bfloat16()
    return out


def _plain_diff_step(s):
    b, heads = s["q"].shape[:2]
    longest = s["case"]["longest"]
    slots = s["slots"].long()
    out = torch.empty_like(s["out"])
    lam = _plain_lambda(s)
    for r in torch.arange(b, device=out.device).split(max(1, (1 << 31) // (heads * 64 * max(1, longest)))):
        k = s["k"][slots[r], :longest].float().view(len(r), longest, heads // 2, 2, 64)
        v = s["v"][slots[r], :longest].float().view(len(r), longest, heads // 2, 128)
        valid = torch.arange(longest, device=out.device) < s["lens"][r, None]
        if s["mask"] is not None:
            valid = valid & s["mask"][slots[r], :longest].bool()
        z = (k * s["q"][r].float().view(len(r), 1, heads // 2, 2, 64)).sum(-1) * 0.125                                  # [r, keys, pairs, 2]
        p = _softmax(z.permute(0, 2, 3, 1), valid[:, None, None])
        x = ((p[:, :, 0] - lam * p[:, :, 1])[:, :, None] @ v.permute(0, 2, 1, 3))[:, :, 0]
        out[r] = _plain_norm(s, x).reshape(len(r), heads, 64).bfloat16()
    return out


def _plain_linear(s):
    seqs, heads = _seqs(s["case"]), s["case"]["heads"]
    D, C = s["q"].shape[2], 256
    cu, g = _offsets(seqs), s["log_decay"].double()
    out, state = torch.empty_like(s["out"]), torch.empty_like(s["state_out"])
    i = torch.arange(C, device=out.device)
    for n_seq, (a, b) in enumerate(zip(cu, cu[1:])):
        n, chunks = b - a, -(-(b - a) // C)

        def tiles(x):
            x = torch.nn.functional.pad(x[a:b].float(), (0, 0, 0, 0, 0, chunks * C - n))
            return x.view(chunks, C, heads, D).permute(2, 0, 1, 3)                                                      # [heads, chunks, C, D]

        q, k, v = tiles(s["q"]), tiles(s["k"]), tiles(s["v"])
        if s["mask"] is not None:
            k = k * torch.nn.functional.pad(s["mask"][a:b].float(), (0, chunks * C - n)).view(1, chunks, C, 1)
        inside = torch.exp(g[:, None, None] * (i[:, None] - i).clamp(min=0)).float() * (i[:, None] >= i)                # [heads, C, C]
        o = (q @ k.transpose(-1, -2) * inside[:, None]) @ v
        adds = (k * torch.exp(g[:, None] * (C - 1 - i)).float()[:, None, :, None]).transpose(-1, -2) @ v                # [heads, chunks, D, D]
        c = torch.arange(chunks, device=out.device)
        across = torch.exp(g[:, None, None] * C * (c[:, None] - 1 - c).clamp(min=0)).float() * (c[:, None] > c)
        before = (across @ adds.flatten(2)).view(heads, chunks, D, D)                                                   # state before each chunk
        if s["state_in"] is not None:
            before += torch.exp(g[:, None] * C * c).float()[..., None, None] * s["state_in"][n_seq][:, None]
        o += torch.exp(g[:, None] * (i + 1)).float()[:, None, :, None] * (q @ before)
        out[a:b] = (s["scale"] * o).permute(1, 2, 0, 3).reshape(chunks * C, heads, D)[:n].bfloat16()
        # the last chunk holds n - C * (chunks - 1) tokens: its end is not the end of a whole chunk
        m = n - C * (chunks - 1)
        tail = (k[:, -1, :m] * torch.exp(g[:, None] * (m - 1 - i[:m])).float()[..., None]).transpose(-1, -2) @ v[:, -1, :m]
        state[n_seq] = torch.exp(g * m).float()[:, None, None] * before[:, -1] + tail
    return {"out": out, "state": state}


def _plain_linear_step(s):
    out, state = s["out"].clone(), s["state_out"].clone()
    rows = (s["slots"] >= 0).nonzero()[:, 0]
    slots = s["slots"][rows].long()
    S = torch.exp(s["log_decay"])[:, None, None] * s["state_in"][slots] + s["k"][rows].float()[..., None] * s["v"][rows].float()[..., None, :]
    out[rows] = (s["scale"] * (s["q"][rows].float()[..., None, :] @ S)[..., 0, :]).bfloat16()
    state[slots] = S
    return {"out": out, "state": state}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, heads = case["op"], case["heads"]
    if op in ("diff", "linear"):
        D, seqs = case.get("head_dim", 64), _seqs(case)
        cu = _offsets(seqs)
        lens = [b - a for a, b in zip(cu, cu[1:])]
        if op == "linear":
            states = (2 if case["carry"] else 1) * len(seqs) * heads * D * D * 4
            return {"bytes": 4 * cu[-1] * heads * D * 2 + states, "flops": 4 * cu[-1] * heads * D * D}
        wanted = [n - int(case["refs"] * (n - text)) for n, (text, *_r) in zip(lens, seqs)]
        keys = [n - ((text - text // 4 if i == 0 else min(1, text)) if case["mask"] else 0) for i, (n, (text, *_r)) in enumerate(zip(lens, seqs))]
        flops = sum(q * k for q, k in zip(wanted, keys)) * (heads // 2) * (2 * 2 * 64 + 2 * 2 * 128)
        return {"bytes": 2 * heads * 64 * sum(2 * q + 2 * k for q, k in zip(wanted, keys)), "flops": flops}
    if op == "diff_step":
        tokens = case["longest"] + (case["batch"] - 1) * (case["shortest"] + case["longest"]) / 2.0      # expected
        if case["mask"]:
            return {"bytes": tokens * (0.9 * heads * 64 * 4 + 1), "flops": 0.9 * tokens * (heads // 2) * 768}
        return {"bytes": tokens * heads * 64 * 4, "flops": tokens * (heads // 2) * 768}
    rows, D = case["batch"] - case["idle"], case["head_dim"]
    return {"bytes": rows * heads * (2 * D * D * 4 + 4 * D * 2), "flops": rows * heads * 4 * D * D}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, heads = case["op"], case["heads"]
    f = torch.float64
    if op in ("diff", "diff_step"):
        a, b, c, d = (x.to(f) for x in s["lams"])
        lam = torch.exp(a.dot(b)) - torch.exp(c.dot(d)) + s["lambda_init"]

        def finish(x):
            if s["gain"] is None:
                return x
            return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * (s["gain"].to(f) * (1.0 - s["lambda_init"]))

        def one_map(q, k, v, valid):
            """q [r, 64], k [n, 64], v [n, 128] in fp64; only the valid keys are there."""
            if not bool(valid.any()):
                return torch.zeros(q.shape[0], 128, dtype=f, device=q.device)
            return torch.softmax(q @ k[valid].T / 8.0, 1) @ v[valid]

    if op == "diff":
        seqs = _seqs(case)
        cu, out = _offsets(seqs), s["out"].to(f)
        for (text, T, H, W), lo, hi in zip(seqs, cu, cu[1:]):
            turn = torch.ones(hi - lo, 32, dtype=torch.complex128, device="cuda")
            grid = torch.cartesian_prod(*(torch.arange(e, dtype=f, device="cuda") for e in (T, H, W))).view(-1, 3)
            at = 0
            for axis, width in enumerate((16, 24, 24)):
                for j in range(width // 2):
                    angle = grid[:, axis] / 10000.0 ** (2.0 * j / width)
                    turn[text:, at] = torch.polar(torch.ones_like(angle), angle)
                    at += 1
            valid = torch.ones(hi - lo, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][lo:hi] != 0
            rows = torch.arange(hi - lo, device="cuda") if s["want"] is None else (s["want"][lo:hi] != 0).nonzero().view(-1)
            for pair in range(heads // 2):
                v = s["v"][lo:hi, 2 * pair: 2 * pair + 2].to(f).reshape(hi - lo, 128)
                q, k = ([torch.view_as_real(torch.view_as_complex(s[x][lo:hi, h].to(f).view(-1, 32, 2)) * turn).view(-1, 64) for h in (2 * pair, 2 * pair + 1)]
                        for x in ("q", "k"))
                for r in rows.split(8192):
                    x = one_map(q[0][r], k[0], v, valid) - lam * one_map(q[1][r], k[1], v, valid)
                    out[lo + r, 2 * pair: 2 * pair + 2] = finish(x).view(-1, 2, 64)
        return out
    if op == "diff_step":
        out = torch.empty(s["out"].shape, dtype=f, device="cuda")
        lens, slots = s["lens"].tolist(), s["slots"].tolist()
        for b, (n, slot) in enumerate(zip(lens, slots)):
            valid = torch.ones(n, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][slot, :n] != 0
            for pair in range(heads // 2):
                v = s["v"][slot, :n, 2 * pair: 2 * pair + 2].to(f).reshape(n, 128)
                q, k = s["q"][b, 2 * pair: 2 * pair + 2].to(f), s["k"][slot, :n, 2 * pair: 2 * pair + 2].to(f)
                x = one_map(q[:1], k[:, 0], v, valid) - lam * one_map(q[1:], k[:, 1], v, valid)
                out[b, 2 * pair: 2 * pair + 2] = finish(x).view(2, 64)
        return out
    g = torch.exp(s["log_decay"].to(f))
    if op == "linear_step":
        out, state = s["out"].to(f), s["state_out"].to(f)
        for b, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                state[slot] = g[:, None, None] * s["state_in"][slot].to(f) + torch.einsum("hk,hv->hkv", s["k"][b].to(f), s["v"][b].to(f))
                out[b] = s["scale"] * torch.einsum("hk,hkv->hv", s["q"][b].to(f), state[slot])
        return {"out": out, "state": state}
    seqs = _seqs(case)
    cu, D = _offsets(seqs), case["head_dim"]
    out = torch.empty(s["out"].shape, dtype=f, device="cuda")
    state = torch.zeros(s["state_out"].shape, dtype=f, device="cuda") if s["state_in"] is None else s["state_in"].to(f)
    for i, (lo, hi) in enumerate(zip(cu, cu[1:])):
        for a in range(lo, hi, 96):                                  # 96 tokens at a time, all heads
            b = min(a + 96, hi)
            q, k, v = (s[x][a:b].to(f).transpose(0, 1) for x in ("q", "k", "v"))
            if s["mask"] is not None:
                k = k * (s["mask"][a:b] != 0).to(f)[:, None]
            t = torch.arange(b - a, dtype=f, device="cuda")
            lag = t[:, None] - t
            w = torch.where(lag >= 0, g[:, None, None] ** lag.clamp(min=0), torch.zeros((), dtype=f, device="cuda"))
            o = torch.bmm(torch.bmm(q, k.mT) * w, v) + torch.bmm(q, state[i]) * (g[:, None] ** (t + 1))[..., None]
            out[a:b] = s["scale"] * o.transpose(0, 1)
            state[i] = state[i] * (g ** (b - a))[:, None, None] + torch.bmm((k * (g[:, None] ** (b - a - 1 - t))[..., None]).mT, v)
    return {"out": out, "state": state}
