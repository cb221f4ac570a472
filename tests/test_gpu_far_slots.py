"""Slots past 32 bits: their pages and places come from a division in 64 bits."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dim", [64, 33])              # on vectors, element by element
@pytest.mark.parametrize("page,pages", [(16, 1 << 29), (7, 1 << 30)])
def test_slots_past_32_bits(dim, page, pages):
    """A cache of 2^33 slots and of 7 * 2^30; its pages share their memory (a page's step is 0), so what can be seen is the
    place in the page, of every slot another one; a slot's page is seen in the next test."""
    store = torch.zeros((2, page, dim), device=DEV)
    caches = [s.as_strided((pages, page, 1, dim), (0, dim, dim, 1), s.storage_offset()) for s in store]
    last = page * pages
    slots = [2 ** 32 + 5, last - 1, last, 2 ** 32, -1]  # the third is past the cache, the fifth is none
    assert len({s % page for s in slots[:2] + slots[3:4]}) == 3
    g = torch.Generator(device=DEV)
    g.manual_seed(page)
    k, v = (torch.randn((len(slots), 1, dim), generator=g, device=DEV) for _ in range(2))
    at = torch.arange(len(slots), dtype=torch.int32, device=DEV)
    freq = torch.rand(dim // 2, generator=g, device=DEV)
    want = torch.zeros_like(store)
    turned = tl.toploc_norm_rotary_prompt(k, k, at, freq)[1]
    for i, s in enumerate(slots):
        if 0 <= s < last:
            want[0, s % page], want[1, s % page] = turned[i, 0], v[i, 0]
    tl.toploc_norm_rotary_paged(k, k, v, at, torch.tensor(slots, device=DEV), freq, *caches)
    assert torch.equal(store, want)


@pytest.mark.parametrize("dim", [8, 3])
def test_pages_past_32_bits_of_slots(dim):
    """Pages of 2^24 tokens that share their memory but for a step of one head: the page of a slot shows in its place."""
    page, pages = 1 << 24, 1 << 9                      # 2^33 slots
    store = torch.zeros((pages + 4, dim), device=DEV)
    cache = store.as_strided((pages, page, 1, dim), (dim, 0, dim, 1))
    slots = [2 ** 32 + 77, 2 ** 33 - 1, 2 ** 32 - 1, 2 ** 33, 5]
    k = torch.arange(1, 6, device=DEV, dtype=torch.float32)[:, None, None].expand(5, 1, dim).contiguous()
    at = torch.zeros(5, dtype=torch.int32, device=DEV)
    tl.toploc_norm_rotary_paged(k, k, k, at, torch.tensor(slots, device=DEV), torch.ones(dim // 2, device=DEV), cache, cache)
    want = torch.zeros_like(store)
    for i, s in enumerate(slots):
        if s < 2 ** 33:
            want[s // page] = i + 1
    assert torch.equal(store, want)
