"""The model-side operators as measured cases: what a serving provider runs around a proof (pages planned
on the GPU, keys and values written to the paged cache, attention of new tokens over it, the norm that
closes a layer) and what a validator runs to recompute the activations (attention over whole packed
prompts, the same norm).

`own` false: the operators' plain form, elementary torch operations in fp32 rounded once at the end.
`own` true: the framework's kernels through the calls a user makes."""
import random

import torch

own = False

DEV = "cuda"
STALE_PAGES = 5      # pages of the cache that belong to nobody: paged addresses never run in order
TAKEN = 7            # entries of the free list that earlier steps have taken
E4M3_MAX = 448.0
SMALLEST_SCALE = 2.0 ** -126


# ---- cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # 64 sequences in lockstep decode (the batch of the 8B-shaped proof benchmark): latency alone counts
        {"name": "plan one step", "op": "plan", "seqs": 64, "cached": 2048, "new": 1, "page": 16, "mix": 1},
        # a validator's intake: a thousand prompts of up to 4096 tokens get their pages at once
        {"name": "plan prompts", "op": "plan", "seqs": 1024, "cached": 0, "new": 4096, "page": 64, "mix": 2},
        # the keys and values of one decode step
        {"name": "write one step", "op": "write", "seqs": 64, "cached": 2048, "new": 1, "page": 16, "kv_heads": 8,
         "head_dim": 128, "mix": 3},
        # the keys and values of a batch of prompts, 65 thousand tokens or so, behind short cached prefixes
        {"name": "write prompts", "op": "write", "seqs": 32, "cached": 500, "new": 4096, "page": 64, "kv_heads": 8,
         "head_dim": 128, "mix": 4},
        # the norm of one decode step at the 8B hidden size, feeding an 8-bit product with a scale per token
        {"name": "norm one step", "op": "norm", "rows": 64, "hidden": 4096, "type": "bfloat16", "group": 0, "mix": 5},
        # the norm of a prefill at the 70B hidden size, 8 bits with a scale per 128 channels
        {"name": "norm prefill", "op": "norm", "rows": 65536, "hidden": 8192, "type": "bfloat16", "group": 128,
         "mix": 6},
        # fp32 activations (the proofs' other type), rows that are no multiple of a vector, no quantisation
        {"name": "norm odd fp32", "op": "norm", "rows": 4095, "hidden": 5001, "type": "float32", "group": -1, "mix": 7},
        # single tokens over the paged cache: one decode step of the 64-sequence batch
        {"name": "paged one token", "op": "paged", "seqs": 64, "cached": 2048, "new": 1, "least": 1, "page": 16,
         "q_heads": 32, "kv_heads": 8, "head_dim": 128, "mix": 8},
        # the proof interval of 32 tokens as one chunk, some sequences idle or with a partial chunk
        {"name": "paged chunks", "op": "paged", "seqs": 24, "cached": 8192, "new": 32, "least": 0, "page": 64,
         "q_heads": 64, "kv_heads": 8, "head_dim": 128, "mix": 9},
        # one long document, a few tokens at a time: few rows, a long axis
        {"name": "paged long context", "op": "paged", "seqs": 1, "cached": 131000, "new": 17, "least": 1, "page": 128,
         "q_heads": 64, "kv_heads": 8, "head_dim": 128, "mix": 10},
        # a validator's batch of short generations of many lengths, packed
        {"name": "prompt short", "op": "prompt", "tokens": 4097, "seqs": 33, "q_heads": 32, "kv_heads": 8,
         "head_dim": 64, "mix": 11},
        # a validator's batch of long generations, packed
        {"name": "prompt long", "op": "prompt", "tokens": 16383, "seqs": 3, "q_heads": 32, "kv_heads": 8,
         "head_dim": 128, "mix": 12},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(("plan", "write", "norm", "paged", "paged", "prompt", "prompt"))
    mix = rng.randrange(1 << 20)
    page = rng.choice((16, 32, 64, 128))
    if op == "plan":
        new = 1 if rng.random() < 0.4 else log(2, 4096)
        return {"op": op, "seqs": log(1, 1024), "cached": log(1, 8192), "new": new, "page": page, "mix": mix}
    if op == "write":
        seqs = log(1, 128)
        new = 1 if rng.random() < 0.4 else log(2, max(3, min(4096, 131072 // seqs)))
        return {"op": op, "seqs": seqs, "cached": log(1, 2048), "new": new, "page": page,
                "kv_heads": rng.choice((1, 2, 4, 8)), "head_dim": rng.choice((64, 128)), "mix": mix}
    if op == "norm":
        hidden = rng.choice((2048, 4096, 8192, log(64, 12000), 8 * log(8, 1500)))
        return {"op": op, "rows": log(1, max(2, 65536 * 8192 // hidden // 2)) if hidden >= 64 else 1, "hidden": hidden,
                "type": rng.choice(("bfloat16", "bfloat16", "float32")), "group": rng.choice((-1, 0, 128)), "mix": mix}
    q_heads, kv_heads = rng.choice(((32, 8), (64, 8), (16, 16), (28, 4), (8, 1)))
    head_dim = rng.choice((64, 128, 128))
    if op == "paged":
        seqs = log(1, 128)
        new = 1 if rng.random() < 0.4 else log(2, 64)
        return {"op": op, "seqs": seqs, "cached": log(16, max(17, min(65536, 262144 // seqs))), "new": new,
                "least": rng.choice((0, 1)) if new > 1 and seqs > 1 else 1, "page": page, "q_heads": q_heads,
                "kv_heads": kv_heads, "head_dim": head_dim, "mix": mix}
    tokens = log(33, int((2.9e9 / (q_heads * head_dim // 64)) ** 0.5))    # up to the largest listed case's work
    return {"op": op, "tokens": tokens, "seqs": rng.randint(1, min(32, tokens)), "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "mix": mix}


def lengths(case):
    """(cached, new) tokens of every sequence: spread evenly up to the case's longest, which is there."""
    r = random.Random(case["mix"])
    n = case["seqs"]
    if case["op"] == "prompt":
        cuts = sorted(r.sample(range(1, case["tokens"]), n - 1))
        ends = cuts + [case["tokens"]]
        return [0] * n, [b - a for a, b in zip([0] + cuts, ends)]
    least = case.get("least", 1)
    cached = [case["cached"] if i == 0 else r.randint(0, case["cached"]) for i in range(n)]
    new = [case["new"] if i == 0 else r.randint(min(least, case["new"]), case["new"]) for i in range(n)]
    return cached, new


def pages_of(tokens, page):
    return -(-tokens // page)


# ---- inputs ----------------------------------------------------------------------------------------

def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def page_table(case, cached, held, g):
    """Pages at random places of the cache: [seqs, width] table of `held` tokens per sequence, -1 elsewhere, the
    pages left over as the free list, and the number of pages of the cache."""
    page = case["page"]
    width = max(pages_of(c + n, page) for c, n in zip(*lengths(case))) + 1
    have = ints([pages_of(h, page) for h in held])
    final = sum(pages_of(c + n, page) for c, n in zip(*lengths(case)))
    total = final + STALE_PAGES + TAKEN
    perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["seqs"], width), -1, dtype=torch.int32, device=DEV)
    mask = torch.arange(width, device=DEV)[None, :] < have[:, None]
    used = sum(pages_of(h, page) for h in held)
    table[mask] = perm[:used]
    return table, perm[used:].contiguous(), total


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + case["mix"])

    def normal(shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)

    op = case["op"]
    state = {"case": dict(case)}
    if op == "norm":
        dtype = getattr(torch, case["type"])
        rows, hidden = case["rows"], case["hidden"]
        # a residual stream with a few massive channels, and a layer's contribution to it
        residual = normal((rows, hidden), dtype).mul_(2.0)
        residual[:, :: max(1, hidden // 4)] *= 40.0
        x = normal((rows, hidden), dtype)
        weight = (1.0 + 0.1 * torch.randn(hidden, generator=g, device=DEV)).to(dtype)
        y_type = dtype if case["group"] < 0 else torch.float8_e4m3fn
        groups = 1 if case["group"] <= 0 else pages_of(hidden, case["group"])
        return {**state, "x": x, "residual": residual, "weight": weight, "residual_out": torch.empty_like(x),
                "y": torch.empty((rows, hidden), dtype=y_type, device=DEV),
                "scales": torch.empty((rows, groups), device=DEV) if case["group"] >= 0 else None}
    cached, new = lengths(case)
    tokens = sum(new)
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    if op == "plan":
        table, free, total = page_table(case, cached, cached, g)
        return {**state, "cached": ints(cached), "new": ints(new), "table": table, "free": free,
                "first": ints([TAKEN]), "tokens": tokens,
                "seq_offsets": torch.empty(len(new) + 1, dtype=torch.int32, device=DEV),
                "kv_lens": torch.empty(len(new), dtype=torch.int32, device=DEV),
                "slots": torch.empty(tokens, dtype=torch.int64, device=DEV),
                "positions": torch.empty(tokens, dtype=torch.int32, device=DEV),
                "next_free": torch.empty(1, dtype=torch.int32, device=DEV),
                "status": torch.empty(len(new), dtype=torch.uint8, device=DEV)}
    dim = case["head_dim"]
    if op == "prompt":
        # queries, keys and values as one projection writes them: views of one tensor
        q_heads, kv_heads = case["q_heads"], case["kv_heads"]
        qkv = normal((tokens, q_heads + 2 * kv_heads, dim))
        qkv[:, q_heads:q_heads + kv_heads, :2] += 3.0            # keys share a direction, as trained ones do
        return {**state, "q": qkv[:, :q_heads], "k": qkv[:, q_heads:q_heads + kv_heads],
                "v": qkv[:, q_heads + kv_heads:], "seq_offsets": ints(offsets), "longest": max(new),
                "out": torch.empty((tokens, q_heads, dim), dtype=torch.bfloat16, device=DEV),
                "lse": torch.empty((tokens, q_heads), device=DEV)}
    kv_heads, page = case["kv_heads"], case["page"]
    kv = [c + n for c, n in zip(cached, new)]
    table, _, total = page_table(case, cached, kv, g)
    k_cache = normal((total, page, kv_heads, dim))
    k_cache[..., :2] += 3.0
    v_cache = normal((total, page, kv_heads, dim))
    if op == "write":
        seq = torch.repeat_interleave(torch.arange(len(new), device=DEV), ints(new, torch.int64))
        pos = ints(cached, torch.int64)[seq] + torch.arange(tokens, device=DEV) - ints(offsets, torch.int64)[seq]
        slots = table[seq, pos // page].to(torch.int64) * page + pos % page
        if tokens > 4:
            slots[tokens // 3] = -1                               # a token that got no page
        return {**state, "k": normal((tokens, kv_heads, dim)), "v": normal((tokens, kv_heads, dim)), "slots": slots,
                "k_cache": k_cache, "v_cache": v_cache}
    return {**state, "q": normal((tokens, case["q_heads"], dim)), "k_cache": k_cache, "v_cache": v_cache,
            "table": table, "seq_offsets": ints(offsets), "kv_lens": ints(kv), "longest": max(new),
            "out": torch.empty((tokens, case["q_heads"], dim), dtype=torch.bfloat16, device=DEV),
            "lse": torch.empty((tokens, case["q_heads"]), device=DEV)}


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    return {"plan": run_plan, "write": run_write, "norm": run_norm, "paged": run_paged, "prompt": run_prompt}[op](state)


def run_plan(s):
    page = s["case"]["page"]
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_plan_pages(s["cached"], s["new"], s["free"], s["first"], s["table"], page, s["seq_offsets"],
                             s["kv_lens"], s["slots"], s["positions"], s["next_free"], s["status"])
        return s["table"], s["seq_offsets"], s["kv_lens"], s["slots"], s["positions"], s["next_free"], s["status"]
    cached, new, free, table = s["cached"].long(), s["new"].long(), s["free"], s["table"]
    n, width = table.shape
    ends = torch.cumsum(new, 0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    before, after = (cached + page - 1) // page, (cached + new + page - 1) // page
    too_wide = after > width
    need = torch.where(too_wide, 0, after - before)
    last = s["first"].long() + torch.cumsum(need, 0)
    first = last - need
    short = (last > free.numel()) & (need > 0)
    fits = ~too_wide & ~short
    status = torch.where(too_wide, 3, torch.where(short, 2, 0)).to(torch.uint8)
    col = torch.arange(width, device=DEV)[None, :]
    fill = (col >= before[:, None]) & (col < after[:, None]) & fits[:, None]
    pick = (first[:, None] + col - before[:, None]).clamp(0, free.numel() - 1)
    table = torch.where(fill, free[pick], table)
    token = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(ends, token, right=True)
    pos = cached[seq] + token - offsets[seq]
    at = table[seq, (pos // page).clamp(max=width - 1)].long()
    slots = torch.where(fits[seq], at * page + pos % page, -1)
    kv = torch.where(fits, cached + new, 0)
    taken = (s["first"].long() + torch.where(fits, need, 0).sum()).int()
    return table, offsets.int(), kv.int(), slots, pos.int(), taken, status


def run_write(s):
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_cache_write(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
        return s["k_cache"], s["v_cache"]
    keep = s["slots"] >= 0
    slots = s["slots"][keep]
    k, v = s["k_cache"], s["v_cache"]
    k.view(-1, *k.shape[2:])[slots] = s["k"][keep]
    v.view(-1, *v.shape[2:])[slots] = s["v"][keep]
    return k, v


def run_norm(s):
    eps, group = 1e-5, s["case"]["group"]
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_rmsnorm_residual(s["x"], s["residual"], s["weight"], eps, residual_out=s["residual_out"], y=s["y"],
                                   scales=s["scales"], group=max(0, group))
        return {"residual": s["residual_out"], "y": s["y"], "scales": s["scales"]}
    h = s["x"].float() + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + eps) * s["weight"].float()
    out = {"residual": h.to(s["x"].dtype), "y": y.to(s["y"].dtype), "scales": None}
    if group >= 0:
        rows, hidden = y.shape
        width = group if group > 0 else hidden
        groups = pages_of(hidden, width)
        padded = y if groups * width == hidden else torch.cat([y, y.new_zeros((rows, groups * width - hidden))], 1)
        parts = padded.view(rows, groups, width)
        scales = (parts.abs().amax(dim=2) / E4M3_MAX).clamp(min=SMALLEST_SCALE)
        q = (parts / scales[:, :, None]).reshape(rows, groups * width)[:, :hidden]
        out["y"], out["scales"] = q.contiguous().to(torch.float8_e4m3fn), scales
    return out


def softmax_of(scores, visible):
    """(weights, their sums, log of the sums of exponentials) of masked scores; rows without a visible key give 0 and
    -inf.  `scores` is overwritten."""
    scores.masked_fill_(~visible, float("-inf"))
    top = scores.amax(dim=-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    weights = scores.sub_(top).exp_()
    total = weights.sum(dim=-1, keepdim=True)
    return weights, total, torch.log(total) + top


def run_paged(s):
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_attention_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["seq_offsets"], s["kv_lens"],
                                  s["longest"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    q, table, kv, t = s["q"], s["table"], s["kv_lens"].long(), s["longest"]
    tokens, q_heads, dim = q.shape
    n, width = table.shape
    page, kv_heads = s["k_cache"].shape[1:3]
    group = q_heads // kv_heads
    starts = s["seq_offsets"].long()[:-1]
    new = s["seq_offsets"].long()[1:] - starts
    row = torch.arange(t, device=DEV)
    rows = (starts[:, None] + row).clamp(max=tokens - 1)
    queries = q[rows].float().view(n, t, kv_heads, group, dim).permute(0, 2, 1, 3, 4)
    queries = queries.reshape(n, kv_heads, t * group, dim)
    pages = table.long().clamp(min=0)
    keys = s["k_cache"][pages].view(n, width * page, kv_heads, dim).permute(0, 2, 1, 3).float()
    values = s["v_cache"][pages].view(n, width * page, kv_heads, dim).permute(0, 2, 1, 3).float()
    scores = torch.matmul(queries, keys.transpose(2, 3)).mul_(dim ** -0.5).view(n, kv_heads, t, group, width * page)
    col = torch.arange(width * page, device=DEV)
    last = (kv - new)[:, None] + row                                        # the newest key a row sees
    visible = (col <= last[:, :, None]) & (col < kv[:, None, None])
    weights, total, lse = softmax_of(scores, visible[:, None, :, None, :])
    out = torch.matmul(weights.view(n, kv_heads, t * group, width * page), values).view(n, kv_heads, t, group, dim)
    out = out / torch.where(total == 0, 1.0, total)
    real = row < new[:, None]
    out = out.permute(0, 2, 1, 3, 4).reshape(n, t, q_heads, dim)[real]
    lse = lse.permute(0, 2, 1, 3, 4).reshape(n, t, q_heads)[real]
    return out.to(q.dtype), lse


def run_prompt(s):
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_attention_prompt(s["q"], s["k"], s["v"], s["seq_offsets"], s["longest"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    q, k, v = s["q"], s["k"], s["v"]
    tokens, q_heads, dim = q.shape
    kv_heads = k.shape[1]
    group = q_heads // kv_heads
    token = torch.arange(tokens, device=DEV)
    seq = torch.searchsorted(s["seq_offsets"].long(), token, right=True)
    visible = (seq[:, None] == seq) & (token[:, None] >= token)
    queries = q.float().view(tokens, kv_heads, group, dim).permute(1, 2, 0, 3).reshape(kv_heads, group * tokens, dim)
    scores = torch.matmul(queries, k.float().permute(1, 2, 0)).mul_(dim ** -0.5)
    weights, total, lse = softmax_of(scores.view(kv_heads, group, tokens, tokens), visible)
    out = torch.matmul(weights.view(kv_heads, group * tokens, tokens), v.float().transpose(0, 1))
    out = out.view(kv_heads, group, tokens, dim) / total
    return (out.permute(2, 0, 1, 3).reshape(tokens, q_heads, dim).to(q.dtype),
            lse.permute(2, 0, 1, 3).reshape(tokens, q_heads))


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "norm":
        rows, hidden = case["rows"], case["hidden"]
        size = 2 if case["type"] == "bfloat16" else 4
        out, scales = (size, 0) if case["group"] < 0 else (1, 4 * (1 if case["group"] == 0 else pages_of(hidden, case["group"])))
        return {"bytes": rows * hidden * (3 * size + out) + rows * scales + hidden * size, "flops": 6 * rows * hidden}
    cached, new = lengths(case)
    tokens = sum(new)
    if op == "plan":
        fresh = sum(pages_of(c + n, case["page"]) - pages_of(c, case["page"]) for c, n in zip(cached, new))
        touched = sum(pages_of(c + n, case["page"]) - c // case["page"] for c, n in zip(cached, new))
        return {"bytes": 12 * tokens + 8 * fresh + 4 * (touched - fresh) + 17 * case["seqs"], "flops": 0}
    dim = case["head_dim"]
    if op == "write":
        return {"bytes": tokens * (8 + 8 * case["kv_heads"] * dim), "flops": 0}
    q_heads, kv_heads = case["q_heads"], case["kv_heads"]
    rows = tokens * q_heads
    keys = sum(c + n for c, n in zip(cached, new) if n > 0)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, new)) * q_heads
    table = 0 if op == "prompt" else 4 * sum(pages_of(c + n, case["page"]) for c, n in zip(cached, new))
    return {"bytes": keys * kv_heads * dim * 4 + rows * (4 * dim + 4) + table + 8 * case["seqs"],
            "flops": 4 * dim * pairs}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op == "plan":
        return None                                               # whole numbers: the plain form's, exactly
    s = prepare(case, seed)
    if op == "norm":
        return exact_norm(s)
    if op == "write":
        out = []
        for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
            flat = cache.double().reshape(-1, new.shape[1] * new.shape[2])
            use = torch.nonzero(s["slots"] >= 0)[:, 0]
            flat.index_copy_(0, s["slots"][use], new.double().reshape(new.shape[0], -1)[use])
            out.append(flat.reshape(cache.shape))
        return tuple(out)
    return exact_attention(s)


def exact_norm(s):
    group = s["case"]["group"]
    x, r, w = s["x"].double(), s["residual"].double(), s["weight"].double()
    h = x + r
    size = (h * h).sum(1) / h.shape[1] + 1e-5
    y = h / torch.sqrt(size)[:, None] * w
    if group < 0:
        return {"residual": h, "y": y, "scales": None}
    width = group if group > 0 else y.shape[1]
    scales = torch.stack([part.abs().max(dim=1).values for part in torch.split(y, width, dim=1)], 1) / E4M3_MAX
    scales = torch.clamp(scales, min=SMALLEST_SCALE)
    q = y / torch.repeat_interleave(scales, width, dim=1)[:, :y.shape[1]]
    return {"residual": h, "y": q, "scales": scales}


def exact_attention(s):
    """Sequence by sequence and head by head, from the definition."""
    case, q = s["case"], s["q"]
    cached, new = lengths(case)
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:2], float("-inf"), dtype=torch.float64, device=DEV)
    at = 0
    for i, (c, n) in enumerate(zip(cached, new)):
        if n == 0:
            continue
        if case["op"] == "prompt":
            k, v = s["k"][at:at + n], s["v"][at:at + n]
        else:
            held = s["table"][i, :pages_of(c + n, case["page"])].long()
            k = s["k_cache"][held].flatten(0, 1)[:c + n]
            v = s["v_cache"][held].flatten(0, 1)[:c + n]
        hidden_keys = torch.arange(c + n, device=DEV)[None, :] > torch.arange(c, c + n, device=DEV)[:, None]
        for h in range(case["kv_heads"]):
            kh, vh = k[:, h].double(), v[:, h].double()
            for head in range(h * group, (h + 1) * group):
                scores = q[at:at + n, head].double() @ kh.T / case["head_dim"] ** 0.5
                scores[hidden_keys] = float("-inf")
                lse[at:at + n, head] = torch.logsumexp(scores, 1)
                out[at:at + n, head] = torch.softmax(scores, 1) @ vh
        at += n
    return out, lse
