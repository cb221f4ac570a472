"""Block tables up to the widest that the header allows, 2^31 - 1 columns: one sequence's row of 8 GB."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
WIDEST = 2 ** 31 - 1


def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def release(table, length, page_size, num_pages, shares=None):
    """One sequence ends whose pages are `taken` off a list that has room for all."""
    n = num_pages
    lens, shares, back = ints([length]), ints([0] * n) if shares is None else shares, torch.full((n,), -7, device=DEV).int()
    out = [ints([-9]), torch.full_like(shares, -9), ints([-9]), ints([99], torch.uint8)]
    tl.toploc_release_pages(ints([1], torch.uint8), lens, table, shares, page_size, back, ints([n]), *out)
    torch.cuda.synchronize()
    return [back] + out


def test_release_of_few_pages():
    table = torch.empty((1, WIDEST), dtype=torch.int32, device=DEV)
    table[0, :4] = ints([6, 2, 9, 4])
    back, lens, shares, head, status = release(table, 50, 16, 12)
    assert status.item() == tl.TOPLOC_SEQ_OK and lens.item() == 0
    assert head.item() == 8 and back.tolist() == [-7] * 8 + [2, 4, 6, 9] and not shares.any()


def test_release_of_a_full_row():
    """Every entry counts, the last one among them: page 0 is held by as many more as the row has it, and is left."""
    n = 1 << 20
    table = torch.arange(WIDEST, dtype=torch.int32, device=DEV).remainder_(n)[None]
    shares = torch.zeros(n, dtype=torch.int32, device=DEV)
    shares[0], shares[n - 1] = 2048, 2047              # 2048 of page 0, 2047 of the last one: one holder is left of either
    back, lens, left, head, status = release(table, WIDEST, 1, n, shares)
    assert status.item() == tl.TOPLOC_SEQ_OK and lens.item() == 0
    assert head.item() == 2 and torch.equal(back[2:], torch.arange(1, n - 1, dtype=torch.int32, device=DEV))
    assert back[:2].tolist() == [-7, -7] and not left.any()


def test_forks_and_compaction_of_few_pages():
    flat = torch.empty((2, WIDEST), dtype=torch.int32, device=DEV)
    flat[0, :3] = ints([5, 1, 8])
    pages = 12
    lens, shares, head = ints([40, 0]), ints([0] * pages), ints([3])
    out = [ints([-9] * s) for s in (2, pages, 2, 2, 1, 1)] + [ints([99, 99], torch.uint8)]
    tl.toploc_fork_pages(ints([-1, 0]), lens, shares, ints([0] * 3 + [7]), head, flat, 16, *out)
    assert out[6].tolist() == [0, 0] and out[0].tolist() == [40, 40] and flat[1, :3].tolist() == [5, 1, 7]
    assert out[2].tolist() == [8, -1] and out[3].tolist() == [7, -1] and out[1].nonzero().flatten().tolist() == [1, 5]
    moved = [torch.empty_like(out[1]), torch.full((pages,), -7, device=DEV).int()]
    moved += [torch.empty_like(out[1]) for _ in range(2)] + [ints([-9]), ints([-9]), ints([99, 99], torch.uint8)]
    tl.toploc_compact_pages(out[0], flat, out[1], 16, flat, *moved)
    assert moved[6].tolist() == [0, 0] and moved[4].item() == 3 and moved[5].item() == 4
    assert moved[2][:3].tolist() == [5, 7, 8] and moved[3][:3].tolist() == [0, 2, 3]
    assert flat[:, :3].tolist() == [[0, 1, 3], [0, 1, 2]] and moved[0].tolist() == [1, 1] + [0] * 10
