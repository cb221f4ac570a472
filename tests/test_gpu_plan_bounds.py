"""The plan of pages where the head of the free list is not an entry of it."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = dict(dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("n", [5, 300])
@pytest.mark.parametrize("first", [-1, -3, -(1 << 31), 9, 1 << 30, (1 << 31) - 1])
def test_no_page_from_a_head_outside_the_list(n, first):
    """Whoever needs a page gets NO_PAGES, whoever does not is planned, and the head stays where it is."""
    page, width = 4, 6
    cached = torch.arange(n, **I32) % 9
    new = torch.ones(n, **I32)
    free = torch.arange(100, 109, **I32)
    table = torch.arange(n * width, **I32).view(n, width)
    before = table.clone()
    offsets, kv = torch.empty(n + 1, **I32), torch.empty(n, **I32)
    slots, positions = torch.empty(n, dtype=torch.int64, device=DEV), torch.empty(n, **I32)
    head, status = torch.empty(1, **I32), torch.empty(n, dtype=torch.uint8, device=DEV)
    tl.toploc_plan_pages(cached, new, free, torch.tensor([first], **I32), table, page, offsets, kv, slots, positions, head,
                         status)
    torch.cuda.synchronize()
    needs = cached % page == 0
    assert torch.equal(status, torch.where(needs, tl.TOPLOC_SEQ_NO_PAGES, tl.TOPLOC_SEQ_OK).to(torch.uint8))
    assert torch.equal(kv, torch.where(needs, 0, cached + 1).to(torch.int32)) and head.item() == first
    assert torch.equal(table, before)
    held = table[torch.arange(n, device=DEV), (cached // page).long()].long() * page + cached % page
    assert torch.equal(slots, torch.where(needs, -1, held)) and torch.equal(positions, cached)
