"""Log probabilities, entropy and alternatives against the definition in 64 bits.

Tolerance, in units of 2^-24.  Of the sum s = sum 2^y relative to itself: a thread adds a partial sum of eight (3 roundings)
per group of eight logits, one after the other, over at most vocab / 2048 + 1 groups; the block's and the row's add 8 + 8
more, rescaling 4; each power is off by 2 units of the instruction, by the rounding of y (0.7 |y|, and |y| p is at most 8 units
where y > 0 and below 1 in sum where it is negative) and by log2 e's own (0.4 |y|): 12.  So lse is off by groups + 40 units, plus
the roundings of the last sums, a few units of |x - max| and of log s each.  The entropy's second sum has the same, relative to
sum p |y| <= sum p (max - x) + 8, and is divided by s."""
import math

import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = 2.0 ** -24
# In the place of infinities in what tolerances are relative to: beyond all numbers of fp32 (one of 4.5e31 is rounded by up to
# 2^-24 4.5e31 = 2.7e24, so nothing smaller will do).
HUGE = 1e39


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def logits_of(g, rows, vocab, dtype, spread=3.0):
    return (torch.randn((rows, vocab), generator=g, device=DEV) * spread).to(dtype)


def check(x, tokens, top, entropy=True, **kw):
    rows, vocab = x.shape
    got = tl.toploc_token_logprobs(x, tokens=tokens, top=top, want_entropy=entropy, **kw)
    x64 = x.double()
    most = x64.amax(1, keepdim=True)
    # from the maximum on: at logits of 2^128 64 bits have steps of 2^75, and log(vocab) would be lost in a log-sum-exp
    p = x64 - most
    p = p - torch.log(p.exp().sum(1, keepdim=True))
    units = vocab // 2048 + 41 + 4 * math.log(vocab)
    far = (most - x64).clamp(max=HUGE)
    if tokens is not None:
        want = p.gather(1, tokens[:, None])[:, 0]
        allowed = UNIT * (units + 4 * far.gather(1, tokens[:, None])[:, 0] + 2 * want.abs().clamp(max=HUGE))
        close(got[0], want, allowed)
    else:
        assert got[0] is None
    if entropy:
        want = -torch.special.xlogy(p.exp(), p.exp()).sum(1)
        spread = (p.exp() * far).sum(1)
        close(got[1], want, UNIT * ((units + 10) * (2 + spread + 8) + 4 * want))
    if top:
        order = torch.sort(x64, dim=1, descending=True, stable=True).indices[:, :top]
        n = order.shape[1]
        want = p.gather(1, order)
        alive = want > -math.inf
        ids = torch.where(alive, order, -1)
        assert torch.equal(got[2][:, :n], ids)
        assert bool((got[2][:, n:] == -1).all()) and bool((got[3][:, n:] == -math.inf).all())
        close(got[3][:, :n], want, UNIT * (units + 4 * far.gather(1, order) + 2 * want.abs().clamp(max=HUGE)))
    return got


def close(got, want, allowed):
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].double(), want[~fine])
    diff = (got.double() - want).abs()[fine]
    assert bool((diff <= allowed[fine]).all()), float((diff / allowed[fine]).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [
    (1, 1), (3, 2), (5, 7), (4, 8), (2, 9), (7, 31), (64, 1000), (1, 128000), (3, 50257), (64, 32000), (65, 8193), (700, 4099),
    (2, 262145), (1, 1 << 20)])
def test_against_64_bits(dtype, rows, vocab):
    g = generator(rows + vocab)
    x = logits_of(g, rows, vocab, dtype)
    tokens = torch.randint(vocab, (rows,), generator=g, device=DEV)
    tokens[0] = vocab - 1
    check(x, tokens, 20)


@pytest.mark.parametrize("top", [0, 1, 2, 3, 5, 8, 9, 31, 32])
def test_numbers_of_alternatives(top):
    g = generator(top)
    for rows, vocab in ((2000, 3000), (3, 64000)):
        check(logits_of(g, rows, vocab, torch.bfloat16), None, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7, 8])
def test_rows_that_begin_anywhere(dtype, offset):
    """Columns of a wider tensor (what lies around a row, NaN here, is not part of it)."""
    g = generator(offset)
    wide = torch.full((9, 5011 + offset), float("nan"), device=DEV).to(dtype)
    x = wide[:, offset:offset + 5003]
    x.copy_(logits_of(g, 9, 5003, dtype))
    check(x, torch.randint(5003, (9,), generator=g, device=DEV), 7)


def test_peaked_and_flat_rows():
    g = generator(1)
    x = logits_of(g, 6, 30000, torch.float32, 1.0)
    x[0, 77] = 60.0                                   # one token has it all
    x[1] = torch.linspace(-90, 90, 30000, device=DEV)          # every logit a new maximum
    x[2] = torch.linspace(90, -90, 30000, device=DEV)
    x[3] *= 40
    x[4] -= 5000
    x[5] += 5000
    check(x, torch.tensor([77, 29999, 0, 5, 6, 7], device=DEV), 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [2, 1000])
def test_equal_logits_go_by_index(dtype, rows):
    """More candidates than the kernel has room for: rows of one value, of two, of a few with long runs."""
    vocab = 20000
    x = torch.zeros((rows, vocab), dtype=dtype, device=DEV)
    x[0, ::3] = -0.0                                           # equal to 0
    x[1, 10000:] = 1.0
    if rows > 2:
        g = generator(2)
        x[2:] = torch.randint(0, 4, (rows - 2, vocab), generator=g, device=DEV).to(dtype)
        x[5] = torch.arange(vocab, device=DEV).div(64, rounding_mode="floor").to(dtype)
    for top in (1, 20, 32):
        check(x, torch.full((rows,), 5, device=DEV), top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_impossible_tokens(dtype):
    g = generator(3)
    inf = float("inf")
    x = logits_of(g, 8, 40000, dtype)
    x[0, 3:] = -inf                                            # three are left
    x[1, :39999] = -inf                                        # the last one
    x[2, 20000:] = -inf
    x[3, ::2] = -inf
    keep = torch.zeros(40000, dtype=torch.bool, device=DEV)
    keep[torch.randint(40000, (400,), generator=g, device=DEV)] = True
    x[4, ~keep] = -inf                                         # one in a hundred
    x[5, 1000:1032] = 50.0
    x[5, :1000] = -inf
    tokens = torch.tensor([2, 39999, 30000, 1, 0, 1010, 5, 6], device=DEV)
    check(x, tokens, 20)
    check(x[:2], tokens[:2], 32)


def test_nothing_is_possible():
    x = torch.full((3, 5000), float("-inf"), device=DEV)
    x[1, 17] = -2.0
    lp, h, ids, alternatives = tl.toploc_token_logprobs(x, torch.tensor([1, 17, 4999], device=DEV), 3, want_entropy=True)
    inf = float("inf")
    assert lp.tolist() == [-inf, 0.0, -inf] and h.tolist() == [0.0, 0.0, 0.0]
    assert ids.tolist() == [[-1] * 3, [17, -1, -1], [-1] * 3]
    assert alternatives.tolist() == [[-inf] * 3, [0.0, -inf, -inf], [-inf] * 3]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 600])
def test_masks_of_the_types_lowest_value(dtype, rows):
    g = generator(4)
    low = torch.finfo(dtype).min
    x = logits_of(g, rows, 9000, dtype)
    x[:, 100:] = low
    check(x, torch.full((rows,), 5, device=DEV), 20)
    x[:] = low                                                 # every token masked: all are equally likely
    check(x, torch.full((rows,), 8999, device=DEV), 4)
    x[0, 5:] = float("-inf")                                   # five of them
    check(x, torch.full((rows,), 4, device=DEV), 7)


def test_logits_out_of_the_products_range():
    """Maxima whose product with log2 e does not fit fp32, of both signs."""
    x = torch.zeros((4, 3000), device=DEV)
    x[0] = 3.3e38
    x[1] = -3.3e38
    x[1, 7] = -3.2e38
    x[2] = torch.linspace(2e29, 3e29, 3000, device=DEV)
    x[3, 5] = 3e38
    x[3, 6:] = -3e38
    tokens = torch.tensor([1, 7, 2999, 5], device=DEV)
    got = tl.toploc_token_logprobs(x, tokens, 2, want_entropy=True)
    assert got[2].tolist() == [[0, 1], [7, 0], [2999, 2998], [5, 0]]
    log = math.log(3000)
    assert abs(got[0][0].item() + log) < 1e-5 and abs(got[1][0].item() - log) < 1e-4
    assert got[0][1:].tolist() == [0.0, 0.0, 0.0] and got[1][1:].tolist() == [0.0, 0.0, 0.0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(5, 100000), (800, 900)])
def test_rows_that_are_not_finite(dtype, rows, vocab):
    """NaN and +inf give NaN to their row alone; the alternatives pass over NaN."""
    g = generator(5)
    x = logits_of(g, rows, vocab, dtype)
    clean = x.clone()
    x[0, 5], x[1, vocab - 1] = float("nan"), float("inf")
    x[2] = float("nan")
    x[3, :-1] = float("-inf")
    x[3, -1] = float("nan")
    tokens = torch.zeros(rows, dtype=torch.int64, device=DEV)
    lp, h, ids, alternatives = tl.toploc_token_logprobs(x, tokens, 5, want_entropy=True)
    assert lp[:4].isnan().all() and h[:4].isnan().all() and alternatives[:4].isnan().all()
    clean[0, 5] = float("-inf")
    order = torch.sort(clean[0].double(), descending=True, stable=True).indices[:5]
    assert torch.equal(ids[0], order)
    assert ids[1, 0].item() == vocab - 1 and (ids[2:4] == -1).all()
    assert lp[4:].isfinite().all() and h[4:].isfinite().all()
    rest = check(clean[4:], tokens[4:], 5)
    assert torch.equal(rest[0], lp[4:]) or rows < 100           # (a row's blocks may be fewer in the larger batch)


def test_tokens_outside_the_vocabulary():
    g = generator(6)
    x = logits_of(g, 5, 777, torch.bfloat16)
    tokens = torch.tensor([-1, 777, 3, -2 ** 63, 2 ** 63 - 1], device=DEV)
    lp = tl.toploc_token_logprobs(x, tokens)[0]
    assert lp.isnan().tolist() == [True, True, False, True, True]


def test_same_inputs_same_bits():
    g = generator(7)
    x = logits_of(g, 300, 60000, torch.bfloat16)
    tokens = torch.randint(60000, (300,), generator=g, device=DEV)
    first = tl.toploc_token_logprobs(x, tokens, 20, want_entropy=True)
    for _ in range(3):
        for a, b in zip(first, tl.toploc_token_logprobs(x, tokens, 20, want_entropy=True)):
            assert torch.equal(a, b)


def test_no_rows_and_given_outputs():
    x = torch.zeros((0, 50), device=DEV)
    lp, h, ids, alternatives = tl.toploc_token_logprobs(x, torch.zeros(0, dtype=torch.int64, device=DEV), 2, True)
    assert lp.shape == h.shape == (0,) and ids.shape == (0, 2)
    g = generator(8)
    x = logits_of(g, 4, 50, torch.float32)
    out = torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    got = tl.toploc_token_logprobs(x, torch.zeros(4, dtype=torch.int64, device=DEV), logprobs=out[0], entropy=out[1])
    assert got[0] is out[0] and got[1] is out[1] and got[2] is None


def test_expanded_rows_and_one_column():
    g = generator(9)
    check(logits_of(g, 300, 1, torch.float32), torch.zeros(300, dtype=torch.int64, device=DEV), 2)
    with pytest.raises(tl.ToplocError):                        # rows that share memory: stride 0 < vocab
        tl.toploc_token_logprobs(logits_of(g, 1, 64, torch.float32).expand(3, 64), top=1)


def test_captured_and_replayed_on_another_stream():
    g = generator(10)
    x = logits_of(g, 4, 40000, torch.bfloat16)
    out = torch.empty((4, 3), dtype=torch.int64, device=DEV), torch.empty((4, 3), device=DEV)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    tl.toploc_token_logprobs(x, top=3)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        tl.toploc_token_logprobs(x, top=3, top_ids=out[0], top_logprobs=out[1])
    for seed in (11, 12):
        x.copy_(logits_of(generator(seed), 4, 40000, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = check(x, None, 3)
        assert torch.equal(out[0], want[2]) and torch.equal(out[1], want[3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,top", [(1, 9, 9), (3, 105047, 5), (700, 1130, 32), (5, 40, 32)])
def test_log_probabilities_of_masked_tokens(dtype, rows, vocab, top):
    """Of tokens at the type's lowest value: their distance from the sum, finite like it, and -inf where that does not fit."""
    g = generator(11)
    low = torch.finfo(dtype).min
    x = logits_of(g, rows, vocab, dtype)
    x[:, min(3, vocab // 3):] = low
    check(x, torch.full((rows,), vocab - 1, device=DEV), top)
    x[0, 0] = -low
    got = tl.toploc_token_logprobs(x[:1], torch.full((1,), vocab - 1, device=DEV), 2)
    assert got[0].item() == -math.inf and got[3][0, 0].item() == 0.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mask", [-1e4, -65504.0, -1e6, -1e7, -2.8e7, -3e7, -1e8, -1e9, -1e10, -1e15, -1e20, -1e29, -1e30, -1e35])
@pytest.mark.parametrize("rows,vocab", [(2, 40000), (900, 3000)])
def test_masks_of_any_size(dtype, mask, rows, vocab):
    """Tokens that a large number is put in the place of, or taken off: in front, behind, everywhere but one, or all."""
    g = generator(12)
    x = logits_of(g, rows, vocab, dtype)
    last = torch.full((rows,), vocab - 1, device=DEV)
    for hide in (slice(0, vocab // 2), slice(100, vocab), slice(0, vocab - 1), slice(0, vocab, 2)):
        y = x.clone()
        y[:, hide] = mask
        check(y, last, 5)
    check(x + mask, last, 5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(3, 30000), (800, 500)])
def test_logits_of_any_size(dtype, rows, vocab):
    g = generator(13)
    x = logits_of(g, rows, vocab, torch.float32, 1.0)
    tokens = torch.randint(vocab, (rows,), generator=g, device=DEV)
    for size in range(0, 38):
        y = (x * 10.0 ** size).clamp(-1.6e38, 1.6e38).to(dtype)
        check(y, tokens, 3)
        y[0] = y[0].abs()
        y[-1] = -y[-1].abs()
        check(y, tokens, 3)
    near = (9.9e6 + 2e5 * torch.rand((rows, vocab), generator=g, device=DEV)).round()
    for sign in (1, -1):                # maxima on both sides of where the kernel sums another way
        check((sign * near).to(dtype), tokens, 3)
