"""What a repeated compaction gives: with a table of its own the same, in place nothing new where the shares follow."""
import numpy as np
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(values, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(values)).to(device=DEV, dtype=dtype)


class Families:
    """Sequences in fours that share their first pages, all over a pool."""

    def __init__(self, seed, seqs, longest, page):
        r = np.random.default_rng(seed)
        lens = r.integers(3 * page, longest + 1, seqs)
        have = -(-lens // page)
        perm, taken = r.permutation(3 * int(have.sum())), 0
        table = np.full((seqs, int(have.max()) + 1), -1)
        for i in range(seqs):
            common = 0 if i % 4 == 0 else min(lens[i], lens[i // 4 * 4]) // page
            table[i, :common] = table[i // 4 * 4, :common]
            table[i, common:have[i]] = perm[taken:taken + have[i] - common]
            taken += have[i] - common
        held = np.concatenate([table[i, :have[i]] for i in range(seqs)])
        self.pages, self.page, self.lens, self.table = len(perm), page, ints(lens), ints(table)
        self.shares = ints(np.maximum(np.bincount(held, minlength=len(perm)) - 1, 0))
        self.seqs = seqs

    def outputs(self):
        out = [torch.full((self.pages,), -9, dtype=torch.int32, device=DEV) for _ in range(4)]
        return out + [ints([-9]), ints([-9]), ints(np.full(self.seqs, 99), torch.uint8)]


@pytest.mark.parametrize("seqs,longest,page", [(8, 100, 16), (300, 400, 8)])
def test_in_place_again_with_the_shares_of_before(seqs, longest, page):
    """The shares go by the table's page numbers: behind a call in place the next one takes what the call before left."""
    p = Families(seqs, seqs, longest, page)
    assert int(p.shares.max()) == 3
    first, second = p.outputs(), p.outputs()
    tl.toploc_compact_pages(p.lens, p.table, p.shares, p.page, p.table, *first)
    table = p.table.clone()
    assert first[4].item() > 0
    tl.toploc_compact_pages(p.lens, p.table, first[0], p.page, p.table, *second)
    assert torch.equal(p.table, table) and second[4].item() == 0 and bool((second[2] == -1).all())
    assert torch.equal(second[0], first[0]) and torch.equal(second[5], first[5]) and not second[6].any()
    held = np.concatenate([r[:n] for r, n in zip(table.cpu().numpy(), -(-p.lens.cpu().numpy() // page))])
    assert np.array_equal(first[0].cpu().numpy(), np.maximum(np.bincount(held, minlength=p.pages) - 1, 0))


def test_captured_in_place_with_the_shares_carried_over():
    """A graph that is replayed hands the shares on itself."""
    p = Families(3, 40, 300, 16)
    out = p.outputs()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tl.toploc_compact_pages(p.lens, p.table, p.shares, p.page, p.table, *out)
        p.shares.copy_(out[0])
    graph.replay()
    torch.cuda.synchronize()
    table, shares = p.table.clone(), p.shares.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p.table, table) and torch.equal(p.shares, shares) and out[4].item() == 0
