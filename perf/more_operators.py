"""More of the model-side operators as measured cases: what happens to queries and keys between a projection and
attention (norm of each head, rotation by position, write to the paged cache), what a sampler and a validator read off
the logits (log probabilities of given tokens, entropy, the likeliest alternatives), and what a paged cache needs beyond
its plan (sequences forked for parallel samples, released when they end, pages compacted so that the pool can shrink).

`own` false: the operators' plain form, elementary torch operations in fp32 (angles of positions in fp64) rounded once at
the end.  `own` true: the framework's kernels through the calls a user makes."""
import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
BASE = 500000.0      # of the rotation's frequencies
STALE_PAGES = 5      # pages of the cache that belong to nobody


# ---- cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # 64 sequences in lockstep decode (the batch of the 8B-shaped proof benchmark): queries and keys of one token each
        # normed and turned, keys and values to the cache; latency alone counts
        {"name": "rotary one step", "op": "rotary", "seqs": 64, "new": 1, "cached": 2048, "q_heads": 32, "kv_heads": 8,
         "head_dim": 128, "turned": 128, "pairs": "halves", "norm": True, "page": 16, "type": "bfloat16", "mix": 1},
        # prompts of up to 4096 tokens on their way into the cache, far positions among them
        {"name": "rotary prompts", "op": "rotary", "seqs": 16, "new": 4096, "cached": 100000, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "turned": 128, "pairs": "halves", "norm": True, "page": 64,
         "type": "bfloat16", "mix": 2},
        # a validator's packed pass (no cache) in fp32, the proofs' other type: neighbouring channels turned, half of a head
        {"name": "rotary packed fp32", "op": "rotary", "seqs": 7, "new": 1001, "cached": 0, "q_heads": 28, "kv_heads": 4,
         "head_dim": 64, "turned": 32, "pairs": "neighbours", "norm": False, "page": 0, "type": "float32", "mix": 3},
        # the logits of one decode step: no given tokens, 20 alternatives, of which the first is the greedy token
        {"name": "logprobs one step", "op": "logprobs", "rows": 64, "vocab": 128000, "top": 20, "given": False,
         "type": "bfloat16", "mix": 4},
        # a validator checks 128 generations of 32 tokens: the given tokens' log probabilities, five alternatives
        {"name": "logprobs generations", "op": "logprobs", "rows": 4097, "vocab": 128000, "top": 5, "given": True,
         "type": "bfloat16", "mix": 5},
        # fp32 logits whose rows begin at odd places, given tokens and entropy only
        {"name": "logprobs odd fp32", "op": "logprobs", "rows": 1000, "vocab": 50257, "top": 0, "given": True,
         "type": "float32", "mix": 6},
        # one prompt sampled eight times over
        {"name": "fork one prompt", "op": "fork", "parents": 1, "fan": 8, "cached": 2047, "page": 16, "caches": 4,
         "kv_heads": 8, "head_dim": 128, "mix": 7},
        # a batch of prompts, eight samples of each: last pages are copied in every layer's caches
        {"name": "fork a batch", "op": "fork", "parents": 64, "fan": 8, "cached": 1001, "page": 32, "caches": 16,
         "kv_heads": 8, "head_dim": 128, "mix": 8},
        # some of the 64 sequences of a decode batch end
        {"name": "release some", "op": "release", "seqs": 64, "family": 1, "cached": 2048, "page": 16, "mix": 9},
        # a large batch of samples in families that share their prompts; half of them end
        {"name": "release families", "op": "release", "seqs": 1024, "family": 8, "cached": 4096, "page": 16, "mix": 10},
        # a small pool after some sequences have ended
        {"name": "compact a small pool", "op": "compact", "seqs": 16, "family": 1, "cached": 2048, "page": 16,
         "caches": 4, "kv_heads": 2, "head_dim": 128, "mix": 11},
        # a large pool with shared prompts, a quarter of its pages in the wrong place
        {"name": "compact a large pool", "op": "compact", "seqs": 256, "family": 4, "cached": 4096, "page": 32,
         "caches": 8, "kv_heads": 2, "head_dim": 128, "mix": 12},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(("rotary", "rotary", "logprobs", "logprobs", "fork", "release", "compact"))
    mix = rng.randrange(1 << 20)
    page = rng.choice((16, 32, 64, 128))
    if op == "rotary":
        q_heads, kv_heads = rng.choice(((32, 8), (64, 8), (16, 16), (28, 4), (8, 1)))
        head_dim = rng.choice((64, 80, 96, 128, 128, 256))
        kind = rng.choice(("bfloat16", "bfloat16", "float32"))
        most = 16 * 4096 * 48 * 128 * 2 // ((q_heads + 2 * kv_heads) * head_dim * (2 if kind == "bfloat16" else 4)) // 2
        seqs = log(1, 128)
        new = 1 if rng.random() < 0.4 else log(2, max(3, most // seqs))
        return {"op": op, "seqs": seqs, "new": new, "cached": rng.choice((0, log(1, 131072))), "q_heads": q_heads,
                "kv_heads": kv_heads, "head_dim": head_dim, "turned": rng.choice((head_dim, head_dim, head_dim // 2)),
                "pairs": rng.choice(("halves", "halves", "neighbours")), "norm": rng.random() < 0.7,
                "page": rng.choice((0, page, page)), "type": kind, "mix": mix}
    if op == "logprobs":
        vocab = rng.choice((32000, 128000, 50257, log(1000, 256000)))
        kind = rng.choice(("bfloat16", "bfloat16", "float32"))
        most = 4097 * 128000 * 2 // (vocab * (2 if kind == "bfloat16" else 4))
        top = rng.choice((0, 1, 5, 20))
        return {"op": op, "rows": log(1, min(most, 8192)), "vocab": vocab, "top": top,
                "given": rng.random() < 0.7 if top else True, "type": kind, "mix": mix}
    if op == "fork":
        parents, fan = log(1, 64), rng.randint(2, 9)
        return {"op": op, "parents": parents, "fan": min(fan, 8) if parents > 32 else fan, "cached": log(16, 1001),
                "page": rng.choice((16, 32)), "caches": rng.choice((2, 4, 8)), "kv_heads": rng.choice((1, 2, 8)),
                "head_dim": rng.choice((64, 128)), "mix": mix}
    family = rng.choice((1, 2, 8))
    if op == "release":
        seqs = log(1, 1024)
        return {"op": op, "seqs": seqs, "family": family, "cached": log(16, min(16384, 4096 * 1024 // seqs)),
                "page": page, "mix": mix}
    seqs = log(2, 256)
    return {"op": op, "seqs": seqs, "family": family, "cached": log(16, min(8192, 4096 * 128 // seqs)), "page": page,
            "caches": rng.choice((2, 4, 8)), "kv_heads": rng.choice((1, 2)), "head_dim": rng.choice((64, 128)),
            "mix": mix}


# ---- what a case's batch looks like ----------------------------------------------------------------

def pages_of(tokens, page):
    return -(-tokens // page)


def tokens_of(case):
    """Rotary: (cached, new) tokens of every sequence, up to the case's longest, which is the first's."""
    r = np.random.default_rng(case["mix"])
    n = case["seqs"]
    cached, new = r.integers(0, case["cached"] + 1, n), r.integers(1, case["new"] + 1, n)
    cached[0], new[0] = case["cached"], case["new"]
    return cached, new


def pool_of(case):
    """Lengths of the sequences (the first the longest), pages each shares with its family's first, and a mask."""
    r = np.random.default_rng(case["mix"])
    if case["op"] == "fork":
        lens = r.integers(1, case["cached"] + 1, case["parents"])
        lens[0] = case["cached"]
        lens = np.concatenate([lens, np.zeros(case["parents"] * (case["fan"] - 1), lens.dtype)])
        return lens, np.zeros_like(lens), r.permutation(np.repeat(np.arange(case["parents"]), case["fan"] - 1))
    n, page = case["seqs"], case["page"]
    lens = r.integers(1, case["cached"] + 1, n)
    lens[0] = case["cached"]
    family = np.arange(n) // case["family"]
    shortest = np.full(family[-1] + 1, case["cached"])
    np.minimum.at(shortest, family, lens)
    common = (shortest // page * 3 // 4)[family] if case["family"] > 1 else np.zeros_like(lens)
    if case["op"] == "compact" and n > 1:
        lens = np.where(r.random(n) < 0.25, 0, lens)     # sequences that have ended: their pages are the holes
        lens[0] = case["cached"]
        common = np.where(lens == 0, 0, common)
    released = r.random(n) < (0.5 if case["family"] > 1 else 0.25)
    released[0] = True
    return lens, common, released


def pages_held(case):
    """Table entries in use and distinct pages of a pool."""
    lens, common, _ = pool_of(case)
    have = pages_of(lens, case["page"])
    if case["op"] == "fork" or case["family"] == 1:
        return int(have.sum()), int(have.sum())
    family = np.arange(len(lens)) // case["family"]
    deepest = np.zeros(family[-1] + 1, common.dtype)
    np.maximum.at(deepest, family, common)
    return int(have.sum()), int((have - common).sum() + deepest.sum())


# ---- inputs ----------------------------------------------------------------------------------------

def on_gpu(values, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(values)).to(device=DEV, dtype=dtype)


def blank(*shape, dtype=torch.int32):
    return torch.full(shape, -1, dtype=dtype, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + case["mix"])

    def normal(shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)

    state = {"case": dict(case)}
    if case["op"] == "rotary":
        return {**state, **prepare_rotary(case, normal, g)}
    if case["op"] == "logprobs":
        return {**state, **prepare_logprobs(case, normal, g)}
    return {**state, **prepare_pool(case, normal, np.random.default_rng((int(seed), case["mix"])))}


def prepare_rotary(case, normal, g):
    kind = getattr(torch, case["type"])
    q_heads, kv_heads, dim = case["q_heads"], case["kv_heads"], case["head_dim"]
    cached, new = tokens_of(case)
    total = int(new.sum())
    seq = np.repeat(np.arange(len(new)), new)
    position = cached[seq] + np.arange(total) - (np.cumsum(new) - new)[seq]
    # queries, keys and values as one projection writes them: views of one tensor
    qkv = normal((total, q_heads + 2 * kv_heads, dim), kind)
    qkv[:, :q_heads + kv_heads, :2] += 3.0                   # a shared direction, as trained ones have
    half = case["turned"] // 2
    s = {"q": qkv[:, :q_heads], "k": qkv[:, q_heads:q_heads + kv_heads], "v": qkv[:, q_heads + kv_heads:],
         "positions": on_gpu(position), "inv_freq": on_gpu(BASE ** (-np.arange(half) / half), torch.float32),
         "q_weight": 1.0 + 0.1 * normal((dim,), kind) if case["norm"] else None,
         "k_weight": 1.0 + 0.1 * normal((dim,), kind) if case["norm"] else None,
         "q_out": torch.empty((total, q_heads, dim), dtype=kind, device=DEV)}
    if case["page"] == 0:
        return {**s, "k_out": torch.empty((total, kv_heads, dim), dtype=kind, device=DEV)}
    page = case["page"]
    first = cached // page                                    # the first page that a sequence's new tokens touch
    count = (cached + new - 1) // page - first + 1
    pages = int(count.sum()) + STALE_PAGES
    held = torch.randperm(pages, generator=g, device=DEV)
    at = on_gpu((np.cumsum(count) - count)[seq] + position // page - first[seq], torch.int64)
    slots = held[at] * page + on_gpu(position % page, torch.int64)
    if total > 4:
        slots[total // 3] = -1                                # a token that got no page
    shape = (pages, page, kv_heads, dim)
    return {**s, "slots": slots, "k_cache": normal(shape, kind), "v_cache": normal(shape, kind)}


def prepare_logprobs(case, normal, g):
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    logits = normal((rows, vocab), getattr(torch, case["type"])).mul_(2.5)
    likely = torch.randint(vocab, (rows, 8), generator=g, device=DEV)
    logits.scatter_add_(1, likely, normal((rows, 8), logits.dtype).abs_().mul_(6.0))   # a few that the model favours
    logits[::7, vocab // 2:] = float("-inf")                  # a grammar allows half of the vocabulary
    pick = torch.randint(8, (rows, 1), generator=g, device=DEV)
    allowed = likely % (vocab // 2)
    tokens = torch.where(torch.arange(rows, device=DEV) % 7 == 0, allowed.gather(1, pick)[:, 0], likely.gather(1, pick)[:, 0])
    return {"logits": logits, "tokens": tokens if case["given"] else None,
            "logprobs": torch.empty(rows, device=DEV) if case["given"] else None,
            "entropy": torch.empty(rows, device=DEV),
            "top_ids": torch.empty((rows, top), dtype=torch.int64, device=DEV) if top else None,
            "top_logprobs": torch.empty((rows, top), device=DEV) if top else None}


def prepare_pool(case, normal, r):
    """Pages at random places of the pool, first ones of a family's sequences shared; one list of all pages, those that
    are taken in front."""
    op, page = case["op"], case["page"]
    lens, common, chosen = pool_of(case)
    n = len(lens)
    have = pages_of(lens, page)
    width = int(have.max()) + 2
    col = np.arange(width)[None, :]
    mask = col < have[:, None]
    family = np.arange(n) // case.get("family", 1)
    deepest = np.zeros(family[-1] + 1, common.dtype)
    np.maximum.at(deepest, family, common)
    shared = mask & (col < common[:, None])
    private = mask & ~shared
    pages = int(private.sum() + deepest.sum())
    spare = (case["parents"] * case["fan"] if op == "fork" else pages // 3) + STALE_PAGES
    perm = r.permutation(pages + spare)
    stock = np.full((len(deepest), width), -1)                # the pages that a family shares
    fill = col < deepest[:, None]
    stock[fill] = perm[:int(deepest.sum())]
    table = np.full((n, width), -1)
    table[private] = perm[int(deepest.sum()):pages]
    table[shared] = stock[family][shared]
    shares = np.maximum(np.bincount(table[mask], minlength=pages + spare) - 1, 0)
    s = {"table": on_gpu(table), "kv_lens": on_gpu(lens), "shares": on_gpu(shares), "free": on_gpu(perm),
         "first": on_gpu([pages]), "kv_lens_out": blank(n), "shares_out": blank(pages + spare), "next": blank(1),
         "status": torch.zeros(n, dtype=torch.uint8, device=DEV)}
    if op == "release":
        return {**s, "release": on_gpu(chosen, torch.uint8)}
    caches = normal((case["caches"], pages + spare, page, case["kv_heads"], case["head_dim"]))
    s = {**s, "caches": caches, "layers": list(caches.unbind(0)), "copies": blank(1)}
    if op == "fork":
        parents = np.concatenate([np.full(case["parents"], -1), chosen])
        return {**s, "parents": on_gpu(parents), "copy_from": blank(n), "copy_to": blank(n)}
    return {**s, "table_out": blank(n, width), "free_out": blank(pages + spare), "copy_from": blank(pages + spare),
            "copy_to": blank(pages + spare)}


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    return {"rotary": run_rotary, "logprobs": run_logprobs, "fork": run_fork, "release": run_release,
            "compact": run_compact}[state["case"]["op"]](state)


def normed(x, weight):
    x = x.float()
    return x if weight is None else x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight.float()


def turned(x, cos, sin, pairs):
    """x with its first channels turned by the angles, in pairs (i, i + half) or (2i, 2i + 1)."""
    half = cos.shape[-1]
    if pairs == "halves":
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], dim=-1)
    a, b, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), rest], dim=-1)


def run_rotary(s):
    pairs = s["case"]["pairs"]
    if own:
        import paper_2501_16007_b200 as tl
        if s["case"]["page"] == 0:
            tl.toploc_norm_rotary_prompt(s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["q_weight"],
                                         k_weight=s["k_weight"], eps=EPS, pairing=pairs, q_out=s["q_out"],
                                         k_out=s["k_out"])
            return s["q_out"], s["k_out"]
        tl.toploc_norm_rotary_paged(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["inv_freq"], s["k_cache"],
                                    s["v_cache"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                    pairing=pairs, q_out=s["q_out"])
        return s["q_out"], s["k_cache"], s["v_cache"]
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = turned(normed(s["q"], s["q_weight"]), cos, sin, pairs).to(s["q"].dtype)
    k = turned(normed(s["k"], s["k_weight"]), cos, sin, pairs).to(s["k"].dtype)
    if s["case"]["page"] == 0:
        return q, k
    keep = s["slots"] >= 0
    slots = s["slots"][keep]
    k_cache, v_cache = s["k_cache"], s["v_cache"]
    k_cache.view(-1, *k.shape[1:])[slots] = k[keep]
    v_cache.view(-1, *k.shape[1:])[slots] = s["v"][keep]
    return q, k_cache, v_cache


def run_logprobs(s):
    top = s["case"]["top"]
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_token_logprobs(s["logits"], tokens=s["tokens"], top=top, logprobs=s["logprobs"], entropy=s["entropy"],
                                 top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])
        return {"logprobs": s["logprobs"], "entropy": s["entropy"], "top_ids": s["top_ids"],
                "top_logprobs": s["top_logprobs"]}
    x = s["logits"].float()
    d = x - x.amax(dim=1, keepdim=True)
    e = d.exp()
    total = e.sum(dim=1)
    entropy = total.log() - torch.where(d == float("-inf"), 0.0, e.mul_(d)).sum(dim=1) / total
    out = {"logprobs": None, "entropy": entropy, "top_ids": None, "top_logprobs": None}
    if s["tokens"] is not None:
        out["logprobs"] = d.gather(1, s["tokens"][:, None])[:, 0] - total.log()
    if top:
        # one key for value and place, so that no two are equal: ties go to the lowest index
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 20) - torch.arange(x.shape[1], device=DEV)
        out["top_ids"] = key.topk(top, dim=1).indices
        out["top_logprobs"] = d.gather(1, out["top_ids"]) - total.log()[:, None]
    return out


def run_fork(s):
    page = s["case"]["page"]
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_fork_pages(s["parents"], s["kv_lens"], s["shares"], s["free"], s["first"], s["table"], page,
                             s["kv_lens_out"], s["shares_out"], s["copy_from"], s["copy_to"], s["copies"], s["next"],
                             s["status"])
        tl.toploc_copy_pages(s["layers"], s["copy_from"], s["copy_to"], s["copies"])
        return (s["table"], s["kv_lens_out"], s["shares_out"], s["copy_from"], s["copy_to"], s["copies"], s["next"],
                s["status"], s["caches"])
    parents, lens, table, free, caches = s["parents"].long(), s["kv_lens"].long(), s["table"], s["free"], s["caches"]
    child, parent = parents >= 0, parents.clamp(min=0)
    length = torch.where(child, lens[parent], 0)
    whole, part = length // page, (length % page > 0).long()
    place = torch.cumsum(part, 0) - part
    fresh = free[s["first"].long() + place].to(table.dtype)
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    inherit = child[:, None] & (col < whole[:, None])
    theirs = table[parent]
    copied = part.bool()
    old = theirs.gather(1, whole[:, None])[:, 0][copied]
    new = fresh[copied]
    out = torch.where(inherit, theirs, torch.where((col == whole[:, None]) & copied[:, None], fresh[:, None], table))
    shares = s["shares"] + torch.bincount(theirs[inherit], minlength=s["shares"].shape[0]).int()
    source, target = torch.full_like(s["parents"], -1), torch.full_like(s["parents"], -1)
    source[:old.shape[0]] = old
    target[:new.shape[0]] = new
    caches[:, new.long()] = caches[:, old.long()]
    copies = part.sum().int()[None]
    return (out, torch.where(child, length, lens).int(), shares, source, target, copies, s["first"] + copies,
            torch.zeros_like(s["status"]), caches)


def run_release(s):
    page = s["case"]["page"]
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_release_pages(s["release"], s["kv_lens"], s["table"], s["shares"], page, s["free"], s["first"],
                                s["kv_lens_out"], s["shares_out"], s["next"], s["status"])
        return s["free"], s["kv_lens_out"], s["shares_out"], s["next"], s["status"]
    gone, lens, table = s["release"].bool(), s["kv_lens"], s["table"]
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    held = gone[:, None] & (col < pages_of(lens, page)[:, None])
    left = s["shares"] - torch.bincount(table[held], minlength=s["shares"].shape[0]).int()
    freed = torch.nonzero(left < 0)[:, 0].int()
    head = s["first"] - freed.shape[0]
    at = torch.arange(freed.shape[0], device=DEV) + head
    free = s["free"].clone()
    free[at] = freed
    return free, torch.where(gone, 0, lens), left.clamp(min=0), head, torch.zeros_like(s["status"])


def run_compact(s):
    page = s["case"]["page"]
    if own:
        import paper_2501_16007_b200 as tl
        tl.toploc_compact_pages(s["kv_lens"], s["table"], s["shares"], page, s["table_out"], s["shares_out"],
                                s["free_out"], s["copy_from"], s["copy_to"], s["copies"], s["next"], s["status"])
        tl.toploc_copy_pages(s["layers"], s["copy_from"], s["copy_to"], s["copies"])
        return (s["table_out"], s["shares_out"], s["free_out"], s["copy_from"], s["copy_to"], s["copies"], s["next"],
                s["status"], s["caches"])
    lens, table, caches = s["kv_lens"], s["table"], s["caches"]
    total = s["shares"].shape[0]
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    held = col < pages_of(lens, page)[:, None]
    live = torch.zeros(total, dtype=torch.bool, device=DEV)
    live[table[held].long()] = True
    count = live.sum()
    number = torch.arange(total, device=DEV)
    old = torch.nonzero(live & (number >= count))[:, 0]
    new = torch.nonzero(~live & (number < count))[:, 0]
    moved = number.clone()
    moved[old] = new
    shares = torch.zeros_like(s["shares"])
    shares[moved[live]] = s["shares"][live]
    out = torch.where(held, moved[table.clamp(min=0).long()].int(), s["table_out"])
    source, target = torch.full_like(s["copy_from"], -1), torch.full_like(s["copy_to"], -1)
    source[:old.shape[0]] = old.int()
    target[:new.shape[0]] = new.int()
    free = torch.where(number >= count, number, s["free_out"]).int()
    caches[:, new] = caches[:, old]
    return (out, shares, free, source, target, torch.full_like(s["copies"], old.shape[0]), count.int()[None],
            torch.zeros_like(s["status"]), caches)


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "rotary":
        total, dim = int(tokens_of(case)[1].sum()), case["head_dim"]
        size = 2 if case["type"] == "bfloat16" else 4
        heads = case["q_heads"] + case["kv_heads"]
        moved = heads + (case["kv_heads"] if case["page"] else 0)
        return {"bytes": total * (moved * dim * size * 2 + (12 if case["page"] else 4)),
                "flops": total * heads * (4 * dim * case["norm"] + 3 * case["turned"])}
    if op == "logprobs":
        rows, vocab, top = case["rows"], case["vocab"], case["top"]
        size = 2 if case["type"] == "bfloat16" else 4
        return {"bytes": rows * (vocab * size + 12 * top + 4 + 12 * case["given"]), "flops": 6 * rows * vocab}
    entries, pages = pages_held(case)
    lens, _, chosen = pool_of(case)
    have = pages_of(lens, case["page"])
    if op == "release":
        gone = int(have[chosen].sum())
        return {"bytes": 4 * gone * 2 + 8 * (pages + pages // 3 + STALE_PAGES) + 10 * case["seqs"], "flops": 0}
    token = case["kv_heads"] * case["head_dim"] * 2 * case["caches"]
    if op == "fork":
        partial = lens % case["page"] > 0
        copies = int(partial[chosen].sum())
        total = pages + case["parents"] * case["fan"] + STALE_PAGES
        # (a parent's last page is read once, however many copies are written)
        used = len(np.unique(chosen[partial[chosen]]))
        return {"bytes": (copies + used) * case["page"] * token + 8 * int(have[chosen].sum()) + 8 * total + 13 * len(lens),
                "flops": 0}
    total = pages + pages // 3 + STALE_PAGES
    moves = pages * (total - pages) // total                  # as many as lie behind the live ones' number
    return {"bytes": 2 * moves * case["page"] * token + 8 * entries + 12 * total + 8 * moves + 5 * case["seqs"], "flops": 0}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "rotary":
        return exact_rotary(prepare(case, seed))
    if case["op"] == "logprobs":
        return exact_logprobs(prepare(case, seed))
    return None                                               # whole numbers and moved values: the plain form's, exactly


def exact_rotary(s):
    """Each pair of channels as a complex number, times e^(i position frequency)."""
    half = s["case"]["turned"] // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       s["positions"].double()[:, None] * s["inv_freq"].double())
    out = []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
        y = x.clone()
        halves = s["case"]["pairs"] == "halves"
        first = slice(0, half) if halves else slice(0, 2 * half, 2)
        second = slice(half, 2 * half) if halves else slice(1, 2 * half, 2)
        for h in range(x.shape[1]):
            z = torch.complex(x[:, h, first], x[:, h, second]) * turn
            y[:, h, first], y[:, h, second] = z.real, z.imag
        out.append(y)
    if s["case"]["page"] == 0:
        return tuple(out)
    use = torch.nonzero(s["slots"] >= 0)[:, 0]
    caches = []
    for cache, new in ((s["k_cache"], out[1]), (s["v_cache"], s["v"].double())):
        flat = cache.double().reshape(-1, *new.shape[1:])
        flat.index_copy_(0, s["slots"][use], new[use])
        caches.append(flat.reshape(cache.shape))
    return out[0], *caches


def exact_logprobs(s):
    """A few rows at a time: their log probabilities, and what follows from them."""
    top, parts = s["case"]["top"], []
    for at in range(0, s["logits"].shape[0], 256):
        x = s["logits"][at:at + 256].double()
        p = x - torch.logsumexp(x, 1, keepdim=True)
        h = -torch.special.xlogy(p.exp(), p.exp()).sum(1)
        given = None if s["tokens"] is None else p.gather(1, s["tokens"][at:at + 256, None])[:, 0]
        parts.append((given, h, torch.sort(p, dim=1, descending=True).values[:, :top] if top else None))
    given, h, tops = ([part[i] for part in parts] for i in range(3))
    return {"logprobs": None if s["tokens"] is None else torch.cat(given), "entropy": torch.cat(h), "top_ids": None,
            "top_logprobs": torch.cat(tops) if top else None}
