"""Log probabilities are never above 0 and entropies never below it, as the definition has them: a caller's
log1p(-exp(logprob)) and sqrt(entropy) stay numbers.  No tolerance: these are signs."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
SHAPES = [(4000, 50), (1000, 4099), (64, 1000), (3, 50000), (1, 128000)]   # one block a row, and clusters


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def assert_in_range(x, tokens, top=4):
    logprob, entropy, _, tops = tl.toploc_token_logprobs(x, tokens, top, want_entropy=True)
    assert bool((logprob <= 0).all()), float(logprob.max())
    assert bool((entropy >= 0).all()), float(entropy.min())
    assert bool((tops <= 0).all()), float(tops.max())
    assert bool((tops[:, 0] == logprob).all())         # the likeliest token is the given one here
    return logprob, entropy


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("hidden", [-float("inf"), "lowest", -300.0])
def test_one_token_has_it_all(dtype, rows, vocab, hidden):
    g = generator(rows + vocab)
    x = torch.full((rows, vocab), torch.finfo(dtype).min if hidden == "lowest" else hidden, device=DEV).to(dtype)
    tokens = torch.randint(vocab, (rows,), generator=g, device=DEV)
    for spread in (1.0, 12.0, 30.0):
        x.scatter_(1, tokens[:, None], (torch.randn((rows, 1), generator=g, device=DEV) * spread).clamp(-90, 90).to(dtype))
        logprob, entropy = assert_in_range(x, tokens)
        # the others' e^-210 and less are nothing beside it: 0 to a power's error (2^-22 of it) and a unit of the logarithm
        assert float(logprob.min()) >= -5 * 2.0 ** -24 and float(entropy.max()) <= 5 * 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_sure_models(dtype, rows, vocab):
    """One token some way above all others: weights of the rest from a tenth to nothing in fp32."""
    g = generator(7 * rows + vocab)
    x = torch.randn((rows, vocab), generator=g, device=DEV)
    tokens = torch.randint(vocab, (rows,), generator=g, device=DEV)
    above = x.amax(1, keepdim=True) + 1 + 40 * torch.rand((rows, 1), generator=g, device=DEV)
    x.scatter_(1, tokens[:, None], above)
    assert_in_range(x.to(dtype), tokens)


def test_one_token_vocabulary():
    x = torch.randn((5000, 1), generator=generator(1), device=DEV) * 20
    assert_in_range(x, torch.zeros(5000, dtype=torch.int64, device=DEV))


def test_far_rows():
    g = generator(2)
    x = torch.full((300, 777), -float("inf"), device=DEV)
    tokens = torch.randint(777, (300,), generator=g, device=DEV)
    for size in (1e5, 9e6, 1.1e7, 1e20):
        x.scatter_(1, tokens[:, None], torch.randn((300, 1), generator=g, device=DEV) * size)
        assert_in_range(x, tokens)


def test_nan_stays():
    x = torch.randn((6, 900), generator=generator(3), device=DEV)
    x[1, 5], x[3, 800], x[4] = float("nan"), float("inf"), float("nan")
    tokens = torch.zeros(6, dtype=torch.int64, device=DEV)
    logprob, entropy, _, tops = tl.toploc_token_logprobs(x, tokens, 3, want_entropy=True)
    spoilt = torch.tensor([False, True, False, True, True, False], device=DEV)
    assert torch.equal(torch.isnan(logprob), spoilt) and torch.equal(torch.isnan(entropy), spoilt)
    assert bool(torch.isnan(tops[spoilt]).all()) and bool((tops[~spoilt] <= 0).all())
