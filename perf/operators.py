"""The attention operators of a conditioned generation step: what is measured of them.

A step of a layer stores the scale's K and V rows into an 8-bit cache (one scale per block of 64 tokens and
head, blocks counted from the first token of a segment), attends to that cache through the plan's windows, and
attends to an encoder's states, in 16 or 32 bits or from an 8-bit cache of their own.

    store     K and V rows of some segments -> codes and block scales
    window    windowed attention on an 8-bit cache
    cross     attention to the first len[b] of kv_len keys
    cross8    the same on an 8-bit cache of one segment

`own` False: elementary torch operations in 32 bits; True: the library's calls.
"""
import math
import random

import torch

own = False

D = 64
BLOCK = 64
VAR256 = (1, 2, 3, 4, 5, 6, 8, 10, 13, 16)
VAR512 = (1, 2, 3, 4, 6, 9, 13, 18, 24, 32)
SM = 0.125


def listed():
    return [
        # the smallest store: the second scale's four tokens of a small batch
        dict(name="store_side2", op="store", scales="256", step=1, B=2, H=16, dtype="bf16", kv_len=0, empty=0),
        # the last scale of the 256 x 256 list, batch and heads of the headline step
        dict(name="store_side16", op="store", scales="256", step=9, B=16, H=30, dtype="bf16", kv_len=0, empty=0),
        # an encoder's states in 32 bits, once per prompt: ragged lengths, one prompt empty
        dict(name="store_encoder_f32", op="store", scales="", step=0, B=16, H=30, dtype="f32", kv_len=333, empty=1),
        # an early generation step: latency
        dict(name="window_side4", op="window", scales="256", step=3, B=16, H=30, radius=3, sink=0),
        # the headline generation step on the 8-bit cache
        dict(name="window_side16", op="window", scales="256", step=9, B=16, H=30, radius=3, sink=0),
        # a whole 512 x 512 sequence at once (scoring, prefill)
        dict(name="window_full_512", op="window", scales="512", step=-1, B=8, H=36, radius=4, sink=0),
        # the first generation step: one query per image, short prompts, one of them empty
        dict(name="cross_token", op="cross", B=16, H=30, Hkv=30, q_len=1, kv_len=77, dtype="bf16", empty=1),
        # the last generation step of 256 x 256 on long prompts
        dict(name="cross_side16", op="cross", B=16, H=30, Hkv=30, q_len=256, kv_len=512, dtype="bf16", empty=0),
        # all rows of a 512 x 512 sequence in 32 bits
        dict(name="cross_full_f32", op="cross", B=2, H=16, Hkv=16, q_len=2240, kv_len=301, dtype="f32", empty=0),
        # the whole 512 x 512 sequence, batch and heads of the larger model
        dict(name="cross_full_512", op="cross", B=8, H=36, Hkv=36, q_len=2240, kv_len=512, dtype="bf16", empty=0),
        # a step of 169 rows on an encoder's 8-bit cache
        dict(name="cross8_side13", op="cross8", B=16, H=30, Hkv=30, q_len=169, kv_len=333, dtype="bf16", empty=1),
        # one token against a long context with shared heads: few rows, a long axis
        dict(name="cross8_long", op="cross8", B=2, H=32, Hkv=8, q_len=1, kv_len=30011, dtype="bf16", empty=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_BYTES = 2.45e8           # of a drawn case: the largest listed one's


def draw(rng):
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= _MOST_BYTES:
            return case


def _draw(rng):
    op = rng.choice(["store", "window", "cross", "cross", "cross8", "cross8"])
    empty = rng.choice([0, 0, 1])
    if op == "store":
        if rng.random() < 0.5:
            return dict(op=op, scales=rng.choice(["256", "512"]), step=rng.randrange(10), B=rng.randint(1, 16),
                        H=rng.randint(1, 36), dtype=rng.choice(["bf16", "f32"]), kv_len=0, empty=0)
        return dict(op=op, scales="", step=0, B=rng.randint(1, 16), H=rng.randint(1, 30),
                    dtype=rng.choice(["bf16", "f32"]), kv_len=_log_int(rng, 1, 2000), empty=empty)
    if op == "window":
        scales = rng.choice(["256", "512"])
        return dict(op=op, scales=scales, step=rng.randint(-1, 9), B=rng.randint(1, 8), H=rng.randint(1, 36),
                    radius=rng.choice([-1, 0, 1, 2, 3, 4, 5, 6]), sink=rng.choice([0, 0, 3]))
    while True:
        H = rng.randint(1, 36)
        Hkv = H if rng.random() < 0.6 else rng.choice([h for h in range(1, H + 1) if H % h == 0])
        c = dict(op=op, B=rng.randint(1, 16), H=H, Hkv=Hkv, q_len=_log_int(rng, 1, 2240), kv_len=_log_int(rng, 1, 32000),
                 dtype=rng.choice(["bf16", "bf16", "f32"]) if op == "cross" else "bf16", empty=empty)
        rate = 16 if c["dtype"] == "f32" else 1               # (matrix products in 32 bits are that much slower)
        if c["B"] * H * c["q_len"] * c["kv_len"] * rate <= 8 * 36 * 2240 * 512:
            return c


def _scales(case):
    return {"256": VAR256, "512": VAR512}[case["scales"]]


def _segments(case):
    if case["op"] in ("cross", "cross8") or not case["scales"]:
        return [case["kv_len"]]
    return [s * s for s in _scales(case)]


def _lens(case):
    """Keys per batch row: from a quarter of the axis to all of it, the first row full, `empty` rows without any."""
    B, n = case["B"], case["kv_len"]
    r = random.Random(1000 * B + n)
    lens = [n] + [r.randint((n + 3) // 4, n) for _ in range(B - 1)]
    for i in range(min(case["empty"], B - 1)):
        lens[B - 1 - i] = 0
    return lens


def _randn(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _block_of_token(segments):
    """Block index of every token, and the number of blocks."""
    out, first = [], 0
    for n in segments:
        out += [first + t // BLOCK for t in range(n)]
        first += (n + BLOCK - 1) // BLOCK
    return torch.tensor(out), first


def _plain_store(x, lens, segments, begin, end, codes, scale):
    """Codes and scales of the segments [begin, end), whose rows are x [B, H, n, 64]."""
    block, _ = _block_of_token(segments)
    lo, hi = sum(segments[:begin]), sum(segments[:end])
    block = block[lo:hi].to(x.device)
    b0, nb = int(block[0]), int(block[-1] - block[0]) + 1
    B, H, n, _ = x.shape
    x = x.float()
    valid = torch.ones(B, n, dtype=torch.bool, device=x.device)
    if lens is not None:
        valid = (lo + torch.arange(n, device=x.device))[None] < lens[:, None]
    mag = torch.where(valid[:, None, :, None], x.abs(), torch.zeros_like(x)).amax(-1)
    amax = torch.zeros(B, H, nb, device=x.device)
    amax.scatter_reduce_(2, (block - b0).expand(B, H, n), mag, "amax")
    # quotients in 64 bits, rounded to 32: the correctly rounded 32-bit quotient, on which a code is decided
    s = (amax.double() / 127.0).float()
    row_s = s[:, :, block - b0][..., None]
    q = torch.where(row_s > 0, (x.double() / row_s.double()).float(), torch.zeros_like(x))
    q = q.round().clamp(-127, 127).to(torch.int8)
    codes[:, :, lo:hi] = torch.where(valid[:, None, :, None], q, codes[:, :, lo:hi])
    any_valid = torch.zeros(B, nb, dtype=torch.int32, device=x.device)
    any_valid.scatter_reduce_(1, (block - b0).expand(B, n), valid.int(), "amax")
    scale[:, :, b0:b0 + nb] = torch.where(any_valid[:, None] > 0, s, scale[:, :, b0:b0 + nb])


def _plain_load(codes, scale, segments):
    block, _ = _block_of_token(segments)
    return codes.float() * scale[:, :, block.to(codes.device)][..., None]


def _mask(scales, step, radius, sink, device):
    """[q tokens, all tokens]: the pairs that the windows keep (step -1: all scales' queries)."""
    qs = range(len(scales)) if step < 0 else [step]
    rows = []
    for k in qs:
        sk = scales[k]
        c = torch.arange(sk, device=device)
        parts = []
        for j, sj in enumerate(scales):
            if j > k:
                parts.append(torch.zeros(sk * sk, sj * sj, dtype=torch.bool, device=device))
            elif j < sink or radius < 0:
                parts.append(torch.ones(sk * sk, sj * sj, dtype=torch.bool, device=device))
            else:
                centre = (2 * c + 1) * sj // (2 * sk)
                near = (torch.arange(sj, device=device)[None] - centre[:, None]).abs() <= radius
                parts.append((near[:, None, :, None] & near[None, :, None, :]).reshape(sk * sk, sj * sj))
        rows.append(torch.cat(parts, 1))
    return torch.cat(rows, 0)


def _inputs(case, seed):
    """The tensors that a program has before the call."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[case.get("dtype", "bf16")]
    B, H, seg = case["B"], case["H"], _segments(case)
    n_blocks = _block_of_token(seg)[1]
    L = sum(seg)
    t = {"segments": seg}

    def cache(heads):
        c = {}
        for name in "kv":
            c[name + "8"] = torch.zeros(B, heads, L, D, dtype=torch.int8, device="cuda")
            c[name + "_scale"] = torch.zeros(B, heads, n_blocks, device="cuda")
        return c

    if case["op"] == "store":
        t["begin"], t["end"] = case["step"], case["step"] + 1
        n = sum(seg[t["begin"]:t["end"]])
        # rows as a projection leaves them, heads inside tokens; V as large as K
        t["k"] = _randn((B, n, H, D), g, dtype).transpose(1, 2)
        t["v"] = _randn((B, n, H, D), g, dtype).transpose(1, 2)
        t["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda") if not case["scales"] else None
        t.update(cache(H))
        return t
    if case["op"] == "window":
        n_q = L if case["step"] < 0 else seg[case["step"]]
        t["q"] = _randn((B, H, n_q, D), g, dtype)
        heads = H
    else:
        t["q"] = _randn((B, case["q_len"], H, D), g, dtype).transpose(1, 2)
        t["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
        heads = case["Hkv"]
    if case["op"] == "cross":
        t["k"] = _randn((B, L, heads, D), g, dtype).transpose(1, 2)
        t["v"] = _randn((B, L, heads, D), g, dtype).transpose(1, 2)
        return t
    t.update(cache(heads))
    for name in "kv":
        x = _randn((B, heads, L, D), g, torch.bfloat16)
        _plain_store(x, None, seg, 0, len(seg), t[name + "8"], t[name + "_scale"])
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    t["case"] = case
    if not own:
        if case["op"] == "window":
            t["mask"] = _mask(_scales(case), case["step"], case["radius"], case["sink"], "cuda")
        return t
    import paper_2411_17178_amd as lv
    t["lv"] = lv
    B, H = case["B"], case["H"]
    if case["op"] != "cross":
        t["cache"] = lv.KV8Cache(t["segments"], t["k8"], t["k_scale"], t["v8"], t["v_scale"])
    if case["op"] == "window":
        k = case["step"]
        t["plan"] = lv.litevar_mask_build(_scales(case), case["radius"], None, case["sink"],
                                          None if k < 0 else (k, k + 1), batch_heads=B * H)
        n = lv.litevar_windowed_attn_kv8_workspace_bytes(t["plan"], B, H)
        t["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    elif case["op"] != "store":
        n = lv.litevar_cross_attn_workspace_bytes(B, H, case["Hkv"], case["q_len"], case["kv_len"])
        t["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return t


def _plain_attention(q, k, v, keep, sm, dtype):
    """softmax(sm q k^T where kept) v in 32 bits; q [B, H, n, 64], k, v [B, Hkv, L, 64], keep broadcasts over
    [B, H, n, L]; a row without a kept key is zero."""
    B, H, n, _ = q.shape
    Hkv, L = k.shape[1], k.shape[2]
    q = q.float().reshape(B, Hkv, H // Hkv * n, D)             # (head h reads kv head h / (H / Hkv))
    s = torch.matmul(q, k.float().transpose(-1, -2).contiguous()).mul_(sm).view(B, H, n, L)
    s.masked_fill_(~keep, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    total = p.sum(-1, keepdim=True)
    v = v.float().contiguous()
    o = torch.matmul(p.view(B, Hkv, H // Hkv * n, L), v).view(B, H, n, D)
    return torch.where(total > 0, o / total, torch.zeros_like(o)).to(dtype)


def run(state):
    t, case = state, state["case"]
    if own:
        lv = t["lv"]
        if case["op"] == "store":
            lv.litevar_kv8_store(t["cache"], t["k"], t["v"], (t["begin"], t["end"]), lens=t["lens"])
            return t["k8"], t["k_scale"], t["v8"], t["v_scale"]
        if case["op"] == "window":
            return lv.litevar_windowed_attn_kv8_fwd(t["plan"], t["q"], t["cache"], SM, workspace=t["workspace"])
        if case["op"] == "cross":
            return lv.litevar_cross_attn_fwd(t["q"], t["k"], t["v"], SM, lens=t["lens"], workspace=t["workspace"])
        return lv.litevar_cross_attn_kv8_fwd(t["q"], t["cache"], SM, lens=t["lens"], workspace=t["workspace"])
    if case["op"] == "store":
        for name in "kv":
            _plain_store(t[name], t["lens"], t["segments"], t["begin"], t["end"], t[name + "8"], t[name + "_scale"])
        return t["k8"], t["k_scale"], t["v8"], t["v_scale"]
    q = t["q"]
    if case["op"] == "cross":
        k, v = t["k"], t["v"]
    else:
        k = _plain_load(t["k8"], t["k_scale"], t["segments"])
        v = _plain_load(t["v8"], t["v_scale"], t["segments"])
    if case["op"] == "window":
        keep = t["mask"]
    else:
        keep = (torch.arange(k.shape[2], device=q.device)[None] < t["lens"][:, None])[:, None, None]
    return _plain_attention(q, k, v, keep, SM, q.dtype)


def _kept_pairs(case):
    """(pairs that the windows keep, keys that some query may see) of one (batch, head)."""
    scales, step = _scales(case), case["step"]
    pairs = 0
    for k in (range(len(scales)) if step < 0 else [step]):
        for j in range(k + 1):
            sk, sj, r = scales[k], scales[j], case["radius"]
            if j < case["sink"] or r < 0:
                pairs += sk * sk * sj * sj
                continue
            line = 0
            for c in range(sk):
                centre = (2 * c + 1) * sj // (2 * sk)
                line += min(centre + r, sj - 1) - max(centre - r, 0) + 1
            pairs += line * line
    top = len(scales) - 1 if step < 0 else step
    return pairs, sum(s * s for s in scales[:top + 1])


def work(case):
    B, H, seg = case["B"], case["H"], _segments(case)
    size = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "store":
        n = seg[case["step"]]
        tokens = sum(_lens(case)) if not case["scales"] else B * n
        blocks = sum((x + BLOCK - 1) // BLOCK for x in _lens(case)) if not case["scales"] else B * ((n + BLOCK - 1) // BLOCK)
        return {"bytes": 2 * H * (tokens * D * (size + 1) + 4 * blocks), "flops": 2 * H * tokens * D * 2}
    if case["op"] == "window":
        pairs, keys = _kept_pairs(case)
        n_q = sum(seg) if case["step"] < 0 else seg[case["step"]]
        return {"bytes": B * H * (n_q * D * 4 + 2 * keys * D + 8 * ((keys + BLOCK - 1) // BLOCK)), "flops": B * H * pairs * 4 * D}
    keys = sum(_lens(case))
    row = D * size if case["op"] == "cross" else D + 4 / BLOCK
    return {"bytes": int(2 * B * H * case["q_len"] * D * size + 2 * case["Hkv"] * keys * row + 4 * B),
            "flops": H * case["q_len"] * keys * 4 * D}


def exact(case, seed):
    """From the definitions, in 64 bits: one (batch row, kv head) at a time."""
    t = _inputs(case, seed)
    B, H, seg = case["B"], case["H"], t["segments"]
    if case["op"] == "store":
        out = []
        lo = sum(seg[:t["begin"]])
        first = sum((n + BLOCK - 1) // BLOCK for n in seg[:t["begin"]])
        for name in "kv":
            scale = t[name + "_scale"].double()
            for b in range(B):
                n = t[name].shape[2] if t["lens"] is None else min(t[name].shape[2], max(0, int(t["lens"][b]) - lo))
                for i in range(0, n, BLOCK):
                    rows = t[name][b, :, i:min(i + BLOCK, n)].double()
                    scale[b, :, first + i // BLOCK] = rows.abs().flatten(1).max(1).values / 127.0
            out += [None, scale]                               # (codes are decided in 32 bits)
        return tuple(out)
    q = t["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    groups = H // (case["Hkv"] if case["op"] != "window" else H)
    if case["op"] == "window":
        keep = _mask(_scales(case), case["step"], case["radius"], case["sink"], q.device)
    if case["op"] != "cross":
        first, row_block = 0, []
        for n in seg:
            row_block.append(first + torch.div(torch.arange(n, device=q.device), BLOCK, rounding_mode="floor"))
            first += -(-n // BLOCK)
        row_block = torch.cat(row_block)
    for b in range(B):
        n = sum(seg) if case["op"] == "window" else int(t["lens"][b])
        if n == 0:
            continue
        for j in range(H // groups):
            if case["op"] == "cross":
                k, v = t["k"][b, j, :n].double(), t["v"][b, j, :n].double()
            else:
                k = t["k8"][b, j, :n].double() * t["k_scale"][b, j].double()[row_block[:n], None]
                v = t["v8"][b, j, :n].double() * t["v_scale"][b, j].double()[row_block[:n], None]
            for h in range(j * groups, (j + 1) * groups):
                s = SM * (q[b, h].double() @ k.t())
                if case["op"] == "window":
                    s = s.masked_fill(~keep, -math.inf)
                out[b, h] = torch.softmax(s, -1) @ v
    return out
