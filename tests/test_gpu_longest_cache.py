"""The longest cache a call may name (2^31 - 4096 keys, all in one page that the table repeats): no key is lost where the keys
are split over blocks."""
import math

import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_every_key_counts():
    page, dim = 4096, 8
    pages = (1 << 31) // page - 1
    caches = [torch.ones((1, page, 1, dim), device=DEV) for _ in range(2)]
    table = torch.zeros((1, pages), dtype=torch.int32, device=DEV)
    q = torch.zeros((1, 1, dim), device=DEV)             # all scores 0: sums of whole numbers, exact in fp32
    lens = torch.tensor([pages * page], dtype=torch.int32, device=DEV)
    offsets = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    out, lse = tl.toploc_attention_paged(q, *caches, table, offsets, lens, 1, want_lse=True)
    # 64 parts of at most 2^25 keys, joined in fp32: a few roundings of the sum of 64 weights and of the logarithm
    assert abs(lse.item() - math.log(pages * page)) < 1e-5          # a 64th of the keys is 0.016
    assert torch.isfinite(out).all()
