"""Norm and rotation of queries and keys against the definition in 64 bits.

Tolerance, from the arithmetic that the header promises: the result is rounded once (half a step, u relative to the value);
before that a turned channel is a cos - b sin in fp32, whose roundings are relative to |a| + |b|: of the norm 2 products,
half of the sum of squares' (a lane adds 16 of a head's at most 256 squares in a row, 5 shuffles: 21 / 2) and 2 units of rsqrt,
of cos and sin 1 unit and the angle's 2^-26 turns (2 pi 2^-26 < 2 units), 2 of the rotation: under 24 units of 2^-24.  The
element-wise kernel adds 8 squares a lane."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def frequencies(pairs, base=10000.0):
    return (base ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / max(pairs, 1))).float()


def wanted(x, weight, positions, inv_freq, pairing, eps):
    """(result, the magnitude that its fp32 roundings are relative to), float64."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    half = inv_freq.shape[0]
    angle = positions.double()[:, None, None] * inv_freq.double()
    cos, sin = angle.cos(), angle.sin()
    i = torch.arange(half, device=x.device)
    first, second = (i, i + half) if pairing == "halves" else (2 * i, 2 * i + 1)
    y, size = x.clone(), x.abs()
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def assert_near(got, want, size):
    diff = (got.double() - want).abs()
    allowed = U[got.dtype] * want.abs() + 24 * 2.0 ** -24 * size * (1 + U[got.dtype]) + 1e-37
    assert bool((diff <= allowed).all()), float((diff / allowed).max())


def check_prompt(tokens, q_heads, kv_heads, dim, turned, pairing, dtype, norm, seed, far=1000, q=None, k=None, eps=1e-6):
    g = generator(seed)
    if q is None:
        q, k = normal(g, (tokens, q_heads, dim), dtype), normal(g, (tokens, kv_heads, dim), dtype)
    positions = torch.randint(0, far, (tokens,), generator=g, device=DEV).to(torch.int32)
    if tokens > 2:
        positions[0], positions[1] = 0, far
    freq = frequencies(turned // 2)
    weights = [(1 + 0.3 * normal(g, (dim,), torch.float32)).to(dtype) if n else None for n in norm]
    before = q.clone(), k.clone()
    got = tl.toploc_norm_rotary_prompt(q, k, positions, freq, q_weight=weights[0], k_weight=weights[1], eps=eps,
                                       pairing=pairing)
    for x, old, weight, y in zip((q, k), before, weights, got):
        assert torch.equal(x, old)
        assert_near(y, *wanted(x, weight, positions, freq, pairing, eps))
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("q_heads,kv_heads,dim,turned", [
    (32, 8, 128, 128), (4, 1, 64, 64), (28, 4, 128, 64), (5, 3, 96, 96), (7, 2, 80, 80), (3, 1, 256, 256),
    (6, 6, 80, 40),       # turned halves of 20 channels: vectors of 4
    (2, 2, 48, 16), (1, 1, 16, 16), (9, 2, 128, 0),   # nothing turns
    (3, 2, 100, 50), (2, 1, 33, 20), (1, 1, 2, 2), (2, 1, 1, 0), (3, 1, 255, 254)])  # element by element
def test_prompt_against_64_bits(dtype, pairing, q_heads, kv_heads, dim, turned):
    check_prompt(37, q_heads, kv_heads, dim, turned, pairing, dtype, (True, True), q_heads * dim + turned)


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 63, 1000, 20011])
def test_token_counts(tokens):
    check_prompt(tokens, 16, 4, 128, 128, "halves", torch.bfloat16, (True, True), tokens)


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
def test_norm_of_either_or_neither(norm):
    for dim, turned in ((128, 128), (33, 32)):
        check_prompt(50, 3, 2, dim, turned, "halves", torch.float32, norm, 3)


def test_far_positions_are_as_exact_as_near_ones():
    """fp32 angles of a billion would be off by 60 turns."""
    for dtype in U:
        check_prompt(300, 4, 2, 64, 64, "halves", dtype, (True, True), 4, far=2 ** 31 - 1)


def test_negative_positions():
    g = generator(5)
    q, k = normal(g, (3, 2, 64), torch.float32), normal(g, (3, 1, 64), torch.float32)
    positions = torch.tensor([-1, -5, -2 ** 31], dtype=torch.int32, device=DEV)
    freq = frequencies(32)
    for y, x in zip(tl.toploc_norm_rotary_prompt(q, k, positions, freq), (q, k)):
        assert_near(y, *wanted(x, None, positions, freq, "halves", 0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_views_of_one_projection_at_any_place(dtype, offset):
    g = generator(6 + offset)
    dim, heads = 64, 8
    flat = normal(g, (100 * (heads * dim + 3 * offset) + offset,), dtype)
    rows = flat[offset:].as_strided((100, heads, dim), (heads * dim + offset, dim, 1))
    check_prompt(100, 6, 2, dim, dim, "halves", dtype, (True, True), 7, q=rows[:, :6], k=rows[:, 6:])


def test_heads_in_front_of_tokens():
    g = generator(8)
    q, k = normal(g, (6, 50, 128), torch.bfloat16).transpose(0, 1), normal(g, (2, 50, 128), torch.bfloat16).transpose(0, 1)
    check_prompt(50, 6, 2, 128, 128, "neighbours", torch.bfloat16, (True, True), 9, q=q, k=k)


@pytest.mark.parametrize("dim,turned", [(128, 128), (128, 64), (33, 32), (40, 20)])
def test_in_place(dim, turned):
    g = generator(10)
    qkv = normal(g, (77, 9, dim), torch.bfloat16)
    q, k = qkv[:, :6], qkv[:, 6:8]
    positions = torch.arange(77, device=DEV, dtype=torch.int32)
    weight = (1 + 0.1 * normal(g, (dim,), torch.float32)).bfloat16()
    freq = frequencies(turned // 2)
    want = tl.toploc_norm_rotary_prompt(q, k, positions, freq, q_weight=weight, k_weight=weight)
    behind = qkv[:, 8:].clone()
    got = tl.toploc_norm_rotary_prompt(q, k, positions, freq, q_weight=weight, k_weight=weight, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, 8:], behind)


def test_values_that_are_not_finite_stay_in_their_head():
    g = generator(11)
    for dim, turned in ((128, 64), (33, 16)):
        q, k = normal(g, (8, 4, dim), torch.float32), normal(g, (8, 2, dim), torch.float32)
        q[2, 1, 3], q[3, 0, dim - 1], k[5, 1, 0] = float("nan"), float("inf"), float("-inf")
        positions = torch.arange(8, device=DEV, dtype=torch.int32) + 1
        freq = frequencies(turned // 2)
        got = tl.toploc_norm_rotary_prompt(q, k, positions, freq)
        for y, x in zip(got, (q, k)):
            want, size = wanted(x, None, positions, freq, "halves", 0)
            touched = ~torch.isfinite(want)
            # the channel and the one it turns with, or the channel alone where it does not turn
            assert torch.equal(touched, ~torch.isfinite(y))
            assert_near(torch.where(touched, 0, y), torch.where(touched, 0, want), torch.where(touched, 0, size))


def test_zero_heads_and_huge_ones():
    q = torch.zeros((4, 2, 64), dtype=torch.float32, device=DEV)
    q[1] = 1e18                                        # squares up to 1e36: their sum fits fp32
    q[2] = 1e-30
    weight = torch.ones(64, device=DEV)
    positions = torch.arange(4, device=DEV, dtype=torch.int32)
    freq = frequencies(32)
    y, _ = tl.toploc_norm_rotary_prompt(q, q[:, :1].clone(), positions, freq, q_weight=weight, k_weight=weight)
    assert_near(y, *wanted(q, weight, positions, freq, "halves", 1e-6))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,turned,pairing,order", [
    (128, 128, "halves", "token"), (64, 32, "neighbours", "head"), (80, 40, "halves", "token"), (33, 32, "halves", "head"),
    (128, 128, "halves", "page")])
def test_paged(dtype, dim, turned, pairing, order):
    """Keys and values at their slots, everything else of the caches as it was; the queries as without a cache."""
    g = generator(12)
    tokens, q_heads, kv_heads, pages, page = 90, 6, 3, 12, 16
    qkv = normal(g, (tokens, q_heads + 2 * kv_heads, dim), dtype)
    q, k, v = qkv.split((q_heads, kv_heads, kv_heads), dim=1)
    caches = []
    for _ in range(2):
        shape = {"token": (pages, page, kv_heads, dim), "head": (pages, kv_heads, page, dim),
                 "page": (page, pages, kv_heads, dim)}[order]
        c = normal(g, shape, dtype)
        caches.append({"token": c, "head": c.transpose(1, 2), "page": c.transpose(0, 1)}[order])
    k_cache, v_cache = caches
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens]
    slots[4], slots[40] = -1, pages * page                     # skipped, both
    positions = torch.randint(0, 5000, (tokens,), generator=g, device=DEV).to(torch.int32)
    weight = [(1 + 0.3 * normal(g, (dim,), torch.float32)).to(dtype) for _ in range(2)]
    freq = frequencies(turned // 2)
    want_q, want_k = tl.toploc_norm_rotary_prompt(q, k, positions, freq, *weight, pairing=pairing)
    want_cache = [c.clone() for c in caches]
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            want_cache[0][s // page, s % page] = want_k[i]
            want_cache[1][s // page, s % page] = v[i]
    got = tl.toploc_norm_rotary_paged(q, k, v, positions, slots, freq, k_cache, v_cache, *weight, pairing=pairing)
    assert torch.equal(got, want_q)
    assert torch.equal(k_cache, want_cache[0]) and torch.equal(v_cache, want_cache[1])


def test_no_tokens():
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    i = torch.empty(0, dtype=torch.int32, device=DEV)
    out = tl.toploc_norm_rotary_prompt(q, q[:, :2], i, frequencies(32))
    assert out[0].shape == (0, 4, 64)


def test_slots_past_32_bits():
    """A cache of 2^33 elements (its pages overlap in memory, so it takes little): the last slots are found."""
    page, pages = 16, 1 << 28                                  # 2^32 slots
    store = torch.zeros(64 * 16, dtype=torch.float32, device=DEV)
    cache = store.as_strided((pages, page, 1, 64), (0, 64, 64, 1))
    k = torch.ones((2, 1, 64), device=DEV)
    slots = torch.tensor([2 ** 32 - 1, 2 ** 32 + 5], device=DEV)   # the second is past the cache
    i = torch.zeros(2, dtype=torch.int32, device=DEV)
    tl.toploc_norm_rotary_paged(k, k, k, i, slots, frequencies(32), cache, cache)
    assert store.view(16, 64)[15].eq(1).all() and store.view(16, 64)[:15].eq(0).all()


def test_captured_and_replayed_on_another_stream():
    g = generator(14)
    q, k = normal(g, (64, 8, 128), torch.bfloat16), normal(g, (64, 2, 128), torch.bfloat16)
    positions = torch.arange(64, device=DEV, dtype=torch.int32)
    freq = frequencies(64)
    want = tl.toploc_norm_rotary_prompt(q, k, positions, freq)
    out = torch.empty_like(q), torch.empty_like(k)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        tl.toploc_norm_rotary_prompt(q, k, positions, freq, q_out=out[0], k_out=out[1])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    positions += 5
    graph.replay()
    torch.cuda.synchronize()
    assert_near(out[0], *wanted(q, None, positions, freq, "halves", 0))
