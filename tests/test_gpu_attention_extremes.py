"""Scores and values near the ends of their range, in every kernel of attention, against the definition in 64 bits."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
U16, U32 = 2.0 ** -8, 2.0 ** -24

# (type, new tokens, heads, key heads): few rows, many rows on the tensor cores, the fp32 units
KERNELS = [(torch.bfloat16, 1, 4, 1), (torch.bfloat16, 2, 4, 1), (torch.bfloat16, 40, 4, 1), (torch.float32, 2, 4, 1)]


def run(dtype, new, heads, kv_heads, k, v, q):
    """out, lse and the definition of both for one sequence of keys k, values v [keys, kv_heads, dim] and rows q."""
    keys, dim, page = k.shape[0], k.shape[2], 16
    pages = -(-keys // page)
    caches = [torch.zeros((pages, page, kv_heads, dim), dtype=dtype, device=DEV) for _ in range(2)]
    for cache, rows in zip(caches, (k, v)):
        cache.view(-1, kv_heads, dim)[:keys] = rows
    i32 = dict(dtype=torch.int32, device=DEV)
    out, lse = tl.toploc_attention_paged(q, *caches, torch.arange(pages, **i32).view(1, -1), torch.tensor([0, new], **i32),
                                         torch.tensor([keys], **i32), new, want_lse=True)
    torch.cuda.synchronize()
    group = heads // kv_heads
    kk, vv = (t.double().repeat_interleave(group, dim=1) for t in (k, v))
    scores = torch.einsum("thd,jhd->thj", q.double(), kk) * dim ** -0.5
    hidden = torch.arange(keys, device=DEV)[None] > torch.arange(keys - new, keys, device=DEV)[:, None]
    scores = torch.where(hidden[:, None], float("-inf"), scores)
    weights = torch.softmax(scores, -1)
    return out.double(), lse.double(), torch.einsum("thj,jhd->thd", weights, vv), torch.logsumexp(scores, -1)


@pytest.mark.parametrize("dtype,new,heads,kv_heads", KERNELS)
@pytest.mark.parametrize("level", [-300.0, -3.0, 300.0])
def test_a_first_tile_of_minus_infinities(dtype, new, heads, kv_heads, level):
    """The first 200 keys' scores are minus infinity, the others' about `level`: they alone count."""
    keys, dim = 500, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    q = torch.ones((new, heads, dim), dtype=dtype, device=DEV)
    k = torch.full((keys, kv_heads, dim), level / 8, dtype=dtype, device=DEV)      # score 64 * level / 8 / 8
    k[:200, :, 0] = float("-inf")
    v = torch.randn((keys, kv_heads, dim), generator=g, device=DEV).to(dtype)
    out, lse, want, want_lse = run(dtype, new, heads, kv_heads, k, v, q)
    u = U16 if dtype == torch.bfloat16 else U32
    # equal scores: equal weights, exact (up to the score's own error, a few fp32 roundings of |level|, that all share)
    assert ((lse - want_lse).abs() <= U32 * (16 + 16 * want_lse.abs()) + U32 * (keys + 16)).all()
    assert ((out - want).abs() <= u * want.abs() + (u + U32 * (keys + 16)) * v.double().abs().mean() * 4).all()


@pytest.mark.parametrize("dtype,new,heads,kv_heads", KERNELS)
@pytest.mark.parametrize("rise", [5.0, 40.0])
def test_large_values_behind_scores_that_rise(dtype, new, heads, kv_heads, rise):
    """Finite results from values of 1e30 whose scores exceed the first tile's by e^rise."""
    keys, dim = 1000, 128
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    q = torch.ones((new, heads, dim), dtype=dtype, device=DEV)
    k = torch.randn((keys, kv_heads, dim), generator=g, device=DEV).mul_(0.25).to(dtype)
    k[200:, :, :64] += rise / 64 * dim ** 0.5
    v = (torch.randn((keys, kv_heads, dim), generator=g, device=DEV) * 1e30).to(dtype)
    out, lse, want, want_lse = run(dtype, new, heads, kv_heads, k, v, q)
    assert torch.isfinite(out).all()
    half = dtype == torch.bfloat16
    # a score is off by dim roundings of its partial sums and a few of its own; a weight by twice that and, for bf16, its
    # own rounding
    score = U32 * ((dim + 4) * k.double().abs().sum(2).max() * dim ** -0.5 + 8)
    weight = 2 * score + U32 * (keys + 16) + (U16 if half else 0)
    scores = torch.einsum("thd,jd->thj", q.double(), k[:, 0].double()) * dim ** -0.5
    hidden = torch.arange(keys, device=DEV)[None] > torch.arange(keys - new, keys, device=DEV)[:, None]
    spread = torch.softmax(torch.where(hidden[:, None], float("-inf"), scores), -1) @ v[:, 0].double().abs()
    assert ((out - want).abs() <= (U16 if half else U32) * want.abs() + 1.05 * weight * spread).all()
    assert ((lse - want_lse).abs() <= 2 * score + U32 * (keys + 16 + 4 * want_lse.abs())).all()
