"""The model-side operators against plain implementations in 64 bits.

Tolerances follow from the arithmetic the header promises: fp32 accumulation, one rounding of the
output to its type, and for bf16 attention the weights rounded to bf16 for the second product.
u = 2^-8 is bf16's rounding unit, 2^-24 that of fp32, 2^-4 that of e4m3 (2^-10 below its normals)."""
import numpy as np
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
U16, U32 = 2.0 ** -8, 2.0 ** -24


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def ints(values, dtype=torch.int32):
    return torch.tensor(list(values), dtype=dtype, device=DEV)


def offsets_of(lens):
    return [0] + list(np.cumsum(lens))


# ---- pages -----------------------------------------------------------------------------------------

def plan_reference(cached, new, free, first, table, page, max_tokens):
    """One sequence after the other, as the header words it."""
    table = table.copy()
    width, n = table.shape[1], len(cached)
    offsets, kv, status = [0], [], []
    slots, positions = np.full(max_tokens, -1, np.int64), np.zeros(max_tokens, np.int32)
    asked = taken = 0
    for i in range(n):
        t = max(new[i], 0)
        begin = offsets[-1] if i == 0 else real_end
        real_end = begin + t
        s, before, need = 0, 0, 0
        if cached[i] < 0 or new[i] < 0:
            s = tl.TOPLOC_SEQ_BAD_LENGTH
        elif real_end > max_tokens:
            s = tl.TOPLOC_SEQ_BATCH_FULL
        elif -(-(cached[i] + t) // page) > width:
            s = tl.TOPLOC_SEQ_TABLE_FULL
        else:
            before = -(-cached[i] // page)
            need = -(-(cached[i] + t) // page) - before
            if need > 0 and first + asked + need > len(free):
                s = tl.TOPLOC_SEQ_NO_PAGES
            else:
                table[i, before:before + need] = free[first + asked:first + asked + need]
                taken += need
            asked += need
        for r in range(t):
            if begin + r < max_tokens:
                pos = cached[i] + r
                positions[begin + r] = pos
                if s == 0 and table[i, pos // page] >= 0:
                    slots[begin + r] = int(table[i, pos // page]) * page + pos % page
        offsets.append(min(real_end, max_tokens))
        kv.append(cached[i] + t if s == 0 else 0)
        status.append(s)
    return table, offsets, kv, slots, positions, first + taken, status


def run_plan(cached, new, free, first, table, page, max_tokens, stream=None):
    n = len(cached)
    t = torch.from_numpy(table).to(DEV)
    out = (torch.full((n + 1,), -9, dtype=torch.int32, device=DEV), torch.full((n,), -9, dtype=torch.int32, device=DEV),
           torch.full((max_tokens,), -9, dtype=torch.int64, device=DEV),
           torch.full((max_tokens,), -9, dtype=torch.int32, device=DEV), ints([-9]),
           torch.full((n,), 99, dtype=torch.uint8, device=DEV))
    args = (ints(cached), ints(new), ints(free), ints([first]), t, page) + out
    torch.cuda.synchronize()
    tl.toploc_plan_pages(*args, stream=stream)
    if stream is None:
        tl.toploc_plan_pages(*args)                      # a repeated call changes nothing
    torch.cuda.synchronize()
    return (t,) + out


def assert_plan(got, want):
    table, offsets, kv, slots, positions, taken, status = got[0], got[1], got[2], got[3], got[4], got[5], got[6]
    assert np.array_equal(table.cpu().numpy(), want[0])
    assert offsets.tolist() == want[1] and kv.tolist() == want[2]
    assert np.array_equal(slots.cpu().numpy(), want[3]) and np.array_equal(positions.cpu().numpy(), want[4])
    assert taken.tolist() == [want[5]] and status.tolist() == want[6]


@pytest.mark.parametrize("n,longest_cached,longest_new,page,width,free,spare", [
    (1, 0, 1, 16, 4, 50, 0),
    (64, 300, 1, 16, 30, 400, 3),       # a decode step
    (7, 100, 0, 16, 20, 10, 0),         # nothing new at all
    (33, 50, 70, 1, 130, 5000, 5),      # a page per token
    (300, 40, 90, 16, 20, 4000, 0),     # more sequences than threads of a block
    (700, 5, 30, 3, 12, 100000, 17),    # pages that are no power of two
    (50, 60, 60, 16, 20, 60, 0),        # the free list runs out
    (40, 100, 100, 16, 8, 1000, 0),     # some rows of the table are too short
    (3, 0, 20000, 64, 400, 2000, 0),    # long prompts
])
def test_plan_pages(n, longest_cached, longest_new, page, width, free, spare):
    r = np.random.default_rng(n * 1000 + page)
    cached = [int(v) for v in r.integers(0, longest_cached + 1, n)]
    cached = [min(c, width * page) for c in cached]
    new = [int(v) for v in r.integers(0, longest_new + 1, n)]
    pages = [int(v) for v in r.permutation(free)]
    table = r.integers(0, 1000, (n, width)).astype(np.int32)
    max_tokens = sum(new) + spare
    want = plan_reference(cached, new, pages, 2, table, page, max_tokens)
    assert_plan(run_plan(cached, new, pages, 2, table, page, max_tokens), want)


def test_plan_pages_conditions():
    cached, new = [5, -1, 3, 4, 0, 7, 16], [3, 2, -4, 1000, 2, 0, 1]
    table = np.arange(7 * 4, dtype=np.int32).reshape(7, 4)
    table[5, 0] = -1
    for max_tokens in (0, 1, 6, 900, 1008, 1100):
        for first, free in ((0, 9), (8, 9), (9, 9), (0, 0), (30, 9)):
            pages = list(range(100, 100 + free))
            want = plan_reference(cached, new, pages, first, table, 4, max_tokens)
            assert_plan(run_plan(cached, new, pages, first, table, 4, max_tokens), want)
    empty = run_plan([], [], [1, 2], 1, np.zeros((0, 4), np.int32), 4, 3)
    assert empty[1].tolist() == [0] and empty[3].tolist() == [-1] * 3 and empty[5].tolist() == [1]


def strided(t, pad):
    """The same values with `pad` elements between rows of the last dimension."""
    wide = torch.empty(t.shape[:-1] + (t.shape[-1] + pad,), dtype=t.dtype, device=t.device)
    view = wide[..., :t.shape[-1]]
    view.copy_(t)
    return view


@pytest.mark.parametrize("tokens,heads,dim,page,dtype,pad,order", [
    (1, 1, 64, 16, torch.bfloat16, 0, "token"),
    (64, 8, 128, 16, torch.bfloat16, 0, "token"),
    (77, 3, 80, 5, torch.float32, 0, "head"),
    (77, 3, 24, 16, torch.bfloat16, 3, "token"),   # rows that are no vectors
    (500, 2, 7, 64, torch.float32, 1, "head"),
    (3000, 8, 128, 64, torch.bfloat16, 8, "head"),
])
def test_cache_write(tokens, heads, dim, page, dtype, pad, order):
    g = generator(tokens + dim)
    pages = -(-tokens // page) + 3
    shape = (pages, page, heads, dim) if order == "token" else (pages, heads, page, dim)
    caches = [strided(normal(g, *shape, dtype=dtype), pad) for _ in range(2)]
    if order == "head":
        caches = [c.transpose(1, 2) for c in caches]
    k, v = (strided(normal(g, tokens, heads, dim, dtype=dtype), pad) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens].contiguous()
    if tokens > 2:
        slots[1] = -1
        slots[2] = pages * page                      # past the cache
    want = [c.clone() for c in caches]
    for w, new in zip(want, (k, v)):
        for t, slot in enumerate(slots.tolist()):
            if 0 <= slot < pages * page:
                w[slot // page, slot % page] = new[t]
    tl.toploc_cache_write(k, v, slots, *caches)
    torch.cuda.synchronize()
    assert torch.equal(caches[0], want[0]) and torch.equal(caches[1], want[1])


# ---- attention -------------------------------------------------------------------------------------

def attention_reference(q, keys, values, first, behind, scale):
    """Rows q [rows, heads, dim] of one sequence against its keys [n, kv_heads, dim]: (out, lse, error bound of out,
    error bound of lse) in 64 bits.  Row r sees keys up to behind + r."""
    rows, heads, dim = q.shape
    n, group = keys.shape[0], heads // keys.shape[1]
    out = torch.zeros((rows, heads, dim), dtype=torch.float64, device=DEV)
    lse = torch.full((rows, heads), float("-inf"), dtype=torch.float64, device=DEV)
    bound, lse_bound = torch.zeros_like(out), torch.zeros_like(lse)
    half = q.dtype == torch.bfloat16
    for r in range(rows):
        count = min(max(behind + r + 1, 0), n)
        if count == 0:
            continue
        for h in range(heads):
            k, v = keys[:count, h // group].double(), values[:count, h // group].double()
            products = q[r, h].double() * k
            s = products.sum(1) * scale
            p = torch.softmax(s, 0)
            out[r, h] = p @ v
            lse[r, h] = torch.logsumexp(s, 0)
            # a score is off by dim roundings of its partial sums and a few of its own; a weight by twice that
            score = U32 * ((dim + 4) * products.abs().sum(1).max() * scale + 8)
            spread = p @ v.abs()
            weights = 2 * score + U32 * (count + 16) + (U16 if half else 0)
            bound[r, h] = (U16 if half else U32) * out[r, h].abs() + 1.05 * weights * spread + 1e-37
            lse_bound[r, h] = 2 * score + U32 * (count + 16 + 4 * lse[r, h].abs())
    return out, lse, bound, lse_bound


def assert_near(got, want, bound, what):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN elsewhere" % what
    same = (got == want) | torch.isnan(want)
    off = torch.where(same, 0.0, (got - want).abs() - bound)
    assert not (off > 0).any(), "%s: off by %g over a bound of %g" % (what, off.max(), bound.max())


def build_cache(g, kv, heads, dim, page, dtype, order="token", pad=0, stale=float("nan")):
    """Caches whose unused places hold `stale`, a table of scattered pages, and every sequence's keys and values."""
    pages = [-(-c // page) for c in kv]
    total, width = sum(pages) + 4, max(pages + [1]) + 1
    shape = (total, page, heads, dim) if order == "token" else (total, heads, page, dim)
    caches = [strided(torch.full(shape, stale, dtype=dtype, device=DEV), pad) for _ in range(2)]
    if order == "head":
        caches = [c.transpose(1, 2) for c in caches]
    table = torch.full((len(kv), width), -1, dtype=torch.int32, device=DEV)
    perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    at, contents = 0, []
    for i, c in enumerate(kv):
        table[i, :pages[i]] = perm[at:at + pages[i]]
        at += pages[i]
        both = [normal(g, c, heads, dim, dtype=dtype) for _ in range(2)]
        for cache, rows in zip(caches, both):
            for j in range(pages[i]):
                part = rows[j * page:(j + 1) * page]
                cache[int(table[i, j]), :part.shape[0]] = part
        contents.append(both)
    return caches, table, contents


def check_paged(kv, new, heads, kv_heads, dim, page, dtype, order="token", pad=0, scale=None, stale=float("nan"),
                seed=0, change=None, max_new=None, extra_rows=0):
    g = generator(seed + 7 * dim + heads)
    caches, table, contents = build_cache(g, kv, kv_heads, dim, page, dtype, order, pad, stale)
    tokens = sum(new) + extra_rows
    q = strided(normal(g, tokens, heads, dim, dtype=dtype), pad)
    if change is not None:
        change(q, caches, table, contents)
    out = strided(torch.full((tokens, heads, dim), 7.0, dtype=dtype, device=DEV), pad)
    lse = torch.full((tokens, heads), 7.0, device=DEV)
    status = torch.zeros(len(kv), dtype=torch.uint8, device=DEV)
    off = offsets_of(new)
    tl.toploc_attention_paged(q, *caches, table, ints(off), ints(kv), max(new) if max_new is None else max_new,
                              scale=scale, out=out, lse=lse, status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * len(kv)
    for i, (k, v) in enumerate(contents):
        rows = slice(off[i], off[i + 1])
        want = attention_reference(q[rows], k, v, off[i], kv[i] - new[i], dim ** -0.5 if scale is None else scale)
        assert_near(out[rows], want[0], want[2], "out of sequence %d" % i)
        assert_near(lse[rows], want[1], want[3], "lse of sequence %d" % i)
    assert (out[off[-1]:] == 7.0).all() and (lse[off[-1]:] == 7.0).all()      # rows of no sequence
    return q, caches, table, out, lse


HEADS = [(4, 1), (3, 3), (14, 2), (16, 2)]


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128),
                                       (torch.bfloat16, 80), (torch.float32, 256), (torch.bfloat16, 8)])
@pytest.mark.parametrize("heads,kv_heads", HEADS)
def test_paged_single_tokens(dtype, dim, heads, kv_heads):
    check_paged([1, 2, 15, 16, 17, 127, 128, 129, 300], [1] * 9, heads, kv_heads, dim, 16, dtype)


@pytest.mark.parametrize("page", [1, 8, 16, 24, 64, 128, 256])
def test_paged_pages_of_every_size(page):
    check_paged([257, 1, 100], [3, 1, 20], 8, 2, 128, page, torch.bfloat16)


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
@pytest.mark.parametrize("order,pad", [("token", 0), ("head", 0), ("token", 8), ("head", 3)])
def test_paged_chunks_orders_and_strides(dtype, dim, order, pad):
    """Chunks of new tokens, idle sequences, whole prompts through the cache, more rows than keys (empty rows)."""
    check_paged([200, 40, 0, 33, 2, 0], [32, 0, 0, 33, 5, 3], 8, 2, dim, 16, dtype, order, pad, extra_rows=2)


def test_paged_odd_groups_and_long_chunks():
    check_paged([300, 131], [150, 131], 7, 1, 128, 32, torch.bfloat16)          # 7 rows a token, tiles that end inside
    check_paged([140], [140], 128, 1, 64, 64, torch.bfloat16, max_new=400)      # the largest group, a loose bound


@pytest.mark.parametrize("scale", [0.01, 3.0])
def test_paged_scales(scale):
    check_paged([500], [4], 8, 2, 64, 16, torch.bfloat16, scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_paged_few_rows_long_axis(dtype):
    """The keys split over blocks and joined; parts that a short sequence leaves empty."""
    kv = [5000, 130, 1]
    q, caches, table, out, lse = check_paged(kv, [1, 1, 1], 8, 2, 128, 64, dtype)
    again = tl.toploc_attention_paged(q, *caches, table, ints([0, 1, 2, 3]), ints(kv), 1, want_lse=True)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)            # the join has one order
    check_paged([6001], [17], 16, 2, 128, 128, dtype)


def test_paged_scores_that_keep_rising():
    """Each tile of keys raises the running maximum by far more than a rounding."""
    def rise(q, caches, table, contents):
        k = contents[0][0]
        q.fill_(1.0)
        k.copy_((torch.arange(k.shape[0], device=DEV) / 40.0).floor()[:, None, None].expand_as(k))
        for j in range(-(-k.shape[0] // 16)):
            part = k[j * 16:(j + 1) * 16]
            caches[0][int(table[0, j]), :part.shape[0]] = part
    check_paged([700], [2], 4, 1, 64, 16, torch.bfloat16, change=rise)
    check_paged([700], [40], 8, 1, 128, 16, torch.bfloat16, change=rise)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_paged_hidden_keys_have_no_influence(bad, dtype):
    """A NaN or infinity in a key or value reaches the rows that see it and no other row."""
    kv, new, page = [150], [40], 16

    def poison(q, caches, table, contents):
        for which, token in ((0, 149), (1, 139), (1, 125)):
            contents[0][which][token, :, 3] = bad
            caches[which][int(table[0, token // page]), token % page, :, 3] = bad

    g = generator(3)
    caches, table, contents = build_cache(g, kv, 2, 64, page, dtype)
    q = normal(g, 40, 8, 64, dtype=dtype)
    poison(q, caches, table, contents)
    out, lse = tl.toploc_attention_paged(q, *caches, table, ints([0, 40]), ints(kv), 40, want_lse=True)
    torch.cuda.synchronize()
    k, v = contents[0]
    clean = attention_reference(q[:39], torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0), 0, 110, 0.125)
    others = [c for c in range(64) if c != 3]
    assert_near(lse[:39], clean[1], clean[3], "lse")
    assert_near(out[:39][..., others], clean[0][..., others], clean[2][..., others], "other channels")
    assert_near(out[:15, :, 3], clean[0][:15, :, 3], clean[2][:15, :, 3], "rows in front of the first")
    seen = out[15:39, :, 3].float()
    assert (torch.isnan(seen) if bad != bad else (seen == bad)).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_paged_hidden_keys_few_rows(dim):
    """The same where a sequence brings few rows."""
    g = generator(17)
    caches, table, contents = build_cache(g, [150], 2, dim, 16, torch.bfloat16)
    q = normal(g, 4, 8, dim)
    for which, token in ((0, 149), (1, 148)):
        contents[0][which][token, :, 5] = float("nan")
        caches[which][int(table[0, token // 16]), token % 16, :, 5] = float("nan")
    out, lse = tl.toploc_attention_paged(q, *caches, table, ints([0, 4]), ints([150]), 4, want_lse=True)
    torch.cuda.synchronize()
    k, v = (torch.nan_to_num(t) for t in contents[0])
    clean = attention_reference(q[:3], k, v, 0, 146, dim ** -0.5)
    others = [c for c in range(dim) if c != 5]
    assert_near(lse[:3], clean[1], clean[3], "lse")
    assert_near(out[:3][..., others], clean[0][..., others], clean[2][..., others], "other channels")
    assert_near(out[:2, :, 5], clean[0][:2, :, 5], clean[2][:2, :, 5], "rows in front of it")
    assert torch.isnan(out[2, :, 5]).all() and torch.isnan(out[3]).all() and torch.isnan(lse[3]).all()


def test_paged_few_rows_without_keys():
    check_paged([0, 5, 1, 3], [1, 2, 2, 0], 8, 2, 128, 16, torch.bfloat16)
    check_paged([0, 5, 1, 3], [1, 4, 6, 0], 4, 4, 64, 32, torch.bfloat16)


@pytest.mark.parametrize("dim,heads,kv_heads,dtype", [(128, 16, 2, torch.bfloat16), (64, 8, 2, torch.bfloat16),
                                                      (128, 8, 2, torch.float32)])
def test_paged_mixture(dim, heads, kv_heads, dtype):
    """Long and short, many rows and one, idle ones between: cuts of the work fall anywhere."""
    check_paged([3000, 70, 1025, 0, 129, 2500], [64, 1, 7, 0, 33, 20], heads, kv_heads, dim, 16, dtype)
    check_paged([4000, 1, 999, 64, 2222], [3, 1, 2, 0, 1], heads, kv_heads, dim, 64, dtype)


def test_paged_cache_beyond_32_bits():
    """Pages whose elements, and slots, lie past 2^31 elements and 2^32 bytes of a cache."""
    page, heads, dim = 16, 8, 128
    pages = (1 << 31) // (page * heads * dim) + 3000
    caches = [torch.empty((pages, page, heads, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    g = generator(23)
    kv, new = 100, 100
    k, v, q = normal(g, kv, heads, dim), normal(g, kv, heads, dim), normal(g, kv, 16, dim)
    chosen = [pages - 1, 5, pages - 2000, pages - 7, 0, pages - 3, 77]
    table = ints([chosen]).view(1, -1)
    at = torch.arange(kv, device=DEV)
    slots = table[0, at // page].to(torch.int64) * page + at % page
    tl.toploc_cache_write(k, v, slots, *caches)
    for cache, rows in zip(caches, (k, v)):
        assert torch.equal(cache[pages - 1, 0], rows[0]) and torch.equal(cache[pages - 2000, 3], rows[2 * page + 3])
    for tokens in (new, 1):
        out, lse = tl.toploc_attention_paged(q[-tokens:], *caches, table, ints([0, tokens]), ints([kv]), tokens,
                                             want_lse=True)
        want = attention_reference(q[-tokens:], k, v, 0, kv - tokens, dim ** -0.5)
        assert_near(out, want[0], want[2], "out")
        assert_near(lse, want[1], want[3], "lse")


def test_paged_promises_that_are_not_kept():
    """Lengths over their bounds and pages outside the cache: flagged, nothing outside is read, the others are right."""
    g = generator(5)
    kv, new = [40, 50, 60], [2, 2, 2]
    caches, table, contents = build_cache(g, kv, 2, 128, 16, torch.bfloat16)
    q = normal(g, 6, 8, 128)
    lens = ints([40, 10 ** 6, -5])
    status = torch.zeros(3, dtype=torch.uint8, device=DEV)
    good = tl.toploc_attention_paged(q, *caches, table, ints([0, 2, 4, 6]), ints(kv), 2)[0]
    out = tl.toploc_attention_paged(q, *caches, table, ints([0, 2, 4, 6]), lens, 2, status=status)[0]
    assert status.tolist()[0] == 0 and status.tolist()[1] in (1, 5) and status.tolist()[2] == 1
    assert torch.equal(out[:2], good[:2])
    table[1, 1], table[2, 0] = 10 ** 6, -7
    status.zero_()
    out = tl.toploc_attention_paged(q, *caches, table, ints([0, 2, 4, 6]), ints(kv), 2, status=status)[0]
    assert status.tolist() == [0, tl.TOPLOC_SEQ_BAD_PAGE, tl.TOPLOC_SEQ_BAD_PAGE]
    assert torch.equal(out[:2], good[:2])
    table[1, 1], table[2, 0] = 0, 0
    status.zero_()
    tl.toploc_attention_paged(q, *caches, table, ints([0, 2, 4, 9]), ints(kv), 2, status=status)
    assert status.tolist()[2] == tl.TOPLOC_SEQ_BAD_LENGTH
    assert "page" not in tl.toploc_sequence_status_string(1) and "cache" in tl.toploc_sequence_status_string(5)


def check_prompt(lens, heads, kv_heads, dim, dtype, fused=True, pad=0, seed=0, max_tokens=None):
    g = generator(seed + dim + heads)
    tokens = sum(lens)
    if fused:
        qkv = normal(g, tokens, heads + 2 * kv_heads, dim, dtype=dtype)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    else:
        q, k, v = (strided(normal(g, tokens, h, dim, dtype=dtype), pad) for h in (heads, kv_heads, kv_heads))
    status = torch.zeros(len(lens), dtype=torch.uint8, device=DEV)
    out, lse = tl.toploc_attention_prompt(q, k, v, ints(offsets_of(lens)), max_tokens or max(lens), want_lse=True,
                                          status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * len(lens)
    for a, b in zip(offsets_of(lens), offsets_of(lens)[1:]):
        want = attention_reference(q[a:b], k[a:b], v[a:b], a, 0, dim ** -0.5)
        assert_near(out[a:b], want[0], want[2], "out of rows %d..%d" % (a, b))
        assert_near(lse[a:b], want[1], want[3], "lse of rows %d..%d" % (a, b))


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64),
                                       (torch.bfloat16, 96)])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (2, 2), (6, 2)])
def test_prompt_lengths(dtype, dim, heads, kv_heads):
    check_prompt([1, 0, 33, 128, 2, 129, 64], heads, kv_heads, dim, dtype)


def test_prompt_long():
    check_prompt([900, 1, 1500], 4, 2, 128, torch.bfloat16)
    check_prompt([1300, 300], 6, 1, 64, torch.bfloat16)


def test_prompt_layouts():
    check_prompt([70, 5], 4, 2, 128, torch.bfloat16, fused=False, pad=8)
    check_prompt([70, 5], 4, 2, 128, torch.bfloat16, fused=False, pad=1)       # rows that are no vectors
    check_prompt([300], 8, 1, 128, torch.bfloat16, max_tokens=1000)
    check_prompt([1], 1, 1, 128, torch.bfloat16)
    check_prompt([31] * 40, 8, 2, 64, torch.bfloat16)


def test_prompt_neighbours_have_no_influence():
    """A prompt full of NaN packed in front of and behind another one."""
    g = generator(11)
    for dtype, dim in ((torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)):
        lens = [37, 61, 45]
        q, k, v = (normal(g, sum(lens), h, dim, dtype=dtype) for h in (8, 2, 2))
        alone = tl.toploc_attention_prompt(q[37:98], k[37:98], v[37:98], ints([0, 61]), 61)[0]
        for t in (q, k, v):
            t[:37] = float("nan")
            t[98:] = float("nan")
        out = tl.toploc_attention_prompt(q, k, v, ints(offsets_of(lens)), 61)[0]
        assert torch.equal(out[37:98], alone) and not torch.isnan(alone).any()


def test_attention_on_another_stream_and_in_a_graph():
    g = generator(13)
    kv, new = [100, 77], [3, 9]
    caches, table, _ = build_cache(g, kv, 2, 128, 16, torch.bfloat16)
    q = normal(g, 12, 8, 128)
    args = (q, *caches, table, ints([0, 3, 12]), ints(kv), 9)
    want = tl.toploc_attention_paged(*args)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.zeros_like(q)
    tl.toploc_attention_paged(*args, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    work = torch.empty(max(16, tl.toploc_attention_workspace_bytes(q, *caches, table, 9)), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tl.toploc_attention_paged(*args, out=out, workspace=work)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


# ---- norm ------------------------------------------------------------------------------------------

def norm_reference(x, r, w, eps):
    h = x.double() + (0 if r is None else r.double())
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.double()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,hidden,pad", [(1, 1, 0), (3, 7, 0), (64, 4096, 0), (5, 8192, 8), (9, 5001, 1),
                                             (2, 1000, 24), (33, 128, 0), (2, 49152, 0), (4, 12296, 0), (700, 2048, 0),
                                             (33, 5001, 0), (3, 16381, 0), (5, 257, 0), (4, 8193, 0)])
@pytest.mark.parametrize("group", [None, 0, 128, 48])
def test_norm(dtype, rows, hidden, pad, group):
    g = generator(rows + hidden)
    x, r = (strided(normal(g, rows, hidden, dtype=dtype) * 3, pad) for _ in range(2))
    w = (1 + 0.1 * torch.randn(hidden, generator=g, device=DEV)).to(dtype)
    if rows > 2:
        x[1], r[1] = 0, 0                                # a row of zeros
    eps = 1e-5
    h, want = norm_reference(x, r, w, eps)
    y, ro, scales = tl.toploc_rmsnorm_residual(x, r, w, eps, quantize=group is not None, group=group or 0)
    torch.cuda.synchronize()
    u = U16 if dtype == torch.bfloat16 else U32
    assert_near(ro, h, u * h.abs() + U32 * h.abs(), "residual")
    # h is off by one fp32 rounding of its terms; mean, root and products by a few, the sum of squares by far fewer
    # than hidden of them
    terms = x.double().abs() + r.double().abs()
    fp32 = U32 * ((8 + hidden / 64) * want.abs() + want.abs() * terms / h.abs().clamp(min=1e-30)) + 1e-38
    if group is None:
        assert_near(y, want, u * want.abs() + fp32 * (1 + u), "y")
        assert scales is None
        return
    width = group or hidden
    parts = torch.split(want, width, dim=1)
    exact = torch.stack([p.abs().amax(1) for p in parts], 1) / 448.0
    exact = exact.clamp(min=2.0 ** -126)
    err = torch.stack([p.amax(1) for p in torch.split(fp32, width, dim=1)], 1) / 448.0
    assert_near(scales, exact, err + 2 * U32 * exact, "scales")
    spread = torch.repeat_interleave(scales.double(), width, dim=1)[:, :hidden]
    stored = y.double() * spread
    # nearest e4m3 of y / scale: half a step, 2^-4 of the value or 2^-10 of the scale
    assert_near(stored, want, torch.maximum(want.abs() * 2.0 ** -4, spread * 2.0 ** -10) * (1 + 1e-3) + 2 * fp32, "y")
    if rows > 2:
        assert not y[1].float().any()


def test_norm_in_place_without_residual_and_special_values():
    g = generator(1)
    for dtype in (torch.bfloat16, torch.float32):
        for hidden in (512, 515):
            x, r = normal(g, 6, hidden, dtype=dtype), normal(g, 6, hidden, dtype=dtype)
            w = normal(g, hidden, dtype=dtype)
            y, ro, _ = tl.toploc_rmsnorm_residual(x, r, w, 1e-6)
            y2, r2, _ = tl.toploc_rmsnorm_residual(x, r, w, 1e-6, residual_out=r)       # in place
            assert r2 is r and torch.equal(r, ro) and torch.equal(y, y2)
            alone, none, _ = tl.toploc_rmsnorm_residual(x, None, w, 1e-6)
            assert none is None
            zero = tl.toploc_rmsnorm_residual(x, torch.zeros_like(x), w, 1e-6)[0]
            assert torch.equal(alone, zero)
            x[2, 5] = float("nan")
            x[3, 7] = float("inf")
            y, _, s = tl.toploc_rmsnorm_residual(x, None, w, 1e-6, quantize=True)
            assert torch.isnan(s[2]).all() and torch.isnan(y[2].float()).all()
            assert torch.isnan(y[3].float())[7] and not torch.isnan(y[[0, 1, 4, 5]].float()).any()
            empty = tl.toploc_rmsnorm_residual(x[:0], None, w, 1e-6)[0]
            assert empty.shape == (0, hidden)
