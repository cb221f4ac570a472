"""The same rows in calls of different sizes: the same ids, numbers within the tolerance of either; the same call, the same bits.
(The number of rows decides how many blocks share a row, and so the order of its sums.)"""
import pytest
import torch

import paper_2501_16007_b200 as tl
from test_gpu_logprobs import check

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1000, 50257, 128000])
def test_rows_of_a_large_call_alone(dtype, vocab):
    g = torch.Generator(device=DEV)
    g.manual_seed(vocab)
    rows = 2000
    x = (torch.randn((rows, vocab), generator=g, device=DEV) * 3).to(dtype)
    tokens = torch.randint(vocab, (rows,), generator=g, device=DEV)
    whole = tl.toploc_token_logprobs(x, tokens, 20, want_entropy=True)
    again = tl.toploc_token_logprobs(x, tokens, 20, want_entropy=True)
    assert all(torch.equal(a, b) for a, b in zip(whole, again))
    for some in (1, 3, 64, 300):
        part = check(x[:some], tokens[:some], 20)
        assert torch.equal(part[2], whole[2][:some])
    # against the call of all rows: twice the tolerance that `check` allows either (logits within 50 of the maximum, log
    # probabilities down to -60, entropies up to 12 with the mean distance from the maximum below 20)
    units = vocab // 2048 + 41 + 48
    for i, allowed in ((0, units + 4 * 50 + 2 * 60), (1, (units + 10) * (2 + 20 + 8) + 4 * 12), (3, units + 4 * 50 + 2 * 60)):
        assert float((part[i].double() - whole[i][:some].double()).abs().max()) <= 2 * allowed * 2.0 ** -24
