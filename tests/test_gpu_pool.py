"""Forks, releases, compaction and copies of pages against plain ones, one sequence after the other as the header words it.
Whole numbers and moved values: everything is compared for equality."""
import numpy as np
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
OK = tl.TOPLOC_SEQ_OK


def ints(values, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(values)).to(device=DEV, dtype=dtype)


def host(t):
    return t.cpu().numpy()


def pages_of(n, page):
    return -(-n // page)


class Pool:
    """A pool with sequences of random lengths, some sharing their first pages, on the host."""

    def __init__(self, seed, seqs, longest, page, family=1, spare=20, empty=0.2, widen=1):
        r = np.random.default_rng(seed)
        self.r, self.page, self.n = r, page, seqs
        self.lens = np.where(r.random(seqs) < empty, 0, r.integers(0, longest + 1, seqs)).astype(np.int32)
        have = pages_of(self.lens, page)
        self.width = int(have.max(initial=0)) + widen
        self.pages = int(have.sum()) + spare
        perm = r.permutation(self.pages).astype(np.int32)
        self.table = r.integers(-5, self.pages + 5, (seqs, self.width)).astype(np.int32)   # what lies behind is anything
        taken = 0
        for i in range(seqs):
            first = i // family * family
            common = 0 if i == first else min(self.lens[i] // page, self.lens[first] // page, r.integers(0, 9))
            self.table[i, :common] = self.table[first, :common]
            self.table[i, common:have[i]] = perm[taken:taken + have[i] - common]
            taken += have[i] - common
        self.free, self.head = perm.copy(), int(taken)
        held = np.concatenate([self.table[i, :have[i]] for i in range(seqs)] + [np.zeros(0, np.int32)])
        self.shares = np.maximum(np.bincount(held, minlength=self.pages) - 1, 0).astype(np.int32)


# ---- forks -----------------------------------------------------------------------------------------

def fork_reference(p, parents, head=None, free=None):
    head = p.head if head is None else head
    free = p.free if free is None else free
    table, kv, shares = p.table.copy(), p.lens.copy(), p.shares.copy()
    source, target, status = np.full(p.n, -1), np.full(p.n, -1), np.zeros(p.n)
    asked = taken = 0
    for i in range(p.n):
        par = parents[i]
        if par < 0:
            continue
        if par >= p.n or parents[par] >= 0:
            status[i] = tl.TOPLOC_SEQ_BAD_PARENT
            continue
        if p.lens[i] != 0:
            status[i] = tl.TOPLOC_SEQ_IN_USE
            continue
        n = int(p.lens[par])
        if n < 0 or pages_of(n, p.page) > p.width:
            status[i] = tl.TOPLOC_SEQ_BAD_LENGTH
            continue
        row = p.table[par, :pages_of(n, p.page)]
        if ((row < 0) | (row >= p.pages)).any():
            status[i] = tl.TOPLOC_SEQ_BAD_PAGE
            continue
        whole = n // p.page
        if n % p.page:
            k, asked = asked, asked + 1
            if head < 0 or head + k >= len(free):
                status[i] = tl.TOPLOC_SEQ_NO_PAGES
                continue
            taken += 1
            page = free[head + k]
            if page < 0 or page >= p.pages:
                status[i] = tl.TOPLOC_SEQ_BAD_PAGE
                continue
            source[k], target[k] = row[whole], page
            table[i, whole] = page
        table[i, :whole] = row[:whole]
        np.add.at(shares, row[:whole], 1)
        kv[i] = n
    return table, kv, shares, source, target, taken, head + taken, status


def run_fork(p, parents, head=None, free=None, repeat=2):
    head = p.head if head is None else head
    n = p.n
    table = ints(p.table)
    out = [ints(np.full(s, -9)) for s in (n, p.pages, n, n, 1, 1)] + [ints(np.full(n, 99), torch.uint8)]
    args = [ints(parents), ints(p.lens), ints(p.shares), ints(p.free if free is None else free), ints([head]), table, p.page]
    for _ in range(repeat):                            # a repeated call changes nothing
        tl.toploc_fork_pages(*args, *out)
    torch.cuda.synchronize()
    return [host(t) for t in [table] + out]


def assert_fork(got, want):
    table, kv, shares, source, target, taken, following, status = want
    assert got[7].tolist() == status.tolist()
    for i in range(len(status)):                       # (the row of a child that was not forked does not count)
        assert status[i] != OK or np.array_equal(got[0][i], table[i]), i
    assert np.array_equal(got[1], kv) and np.array_equal(got[2], shares)
    assert np.array_equal(got[3], source) and np.array_equal(got[4], target)
    assert got[5].tolist() == [taken] and got[6].tolist() == [following]


def children(p, share=0.6):
    """Some of the empty sequences become children of those that are none."""
    parents = np.full(p.n, -1)
    able = np.nonzero(p.lens > 0)[0]
    for i in np.nonzero(p.lens == 0)[0]:
        if len(able) and p.r.random() < share:
            parents[i] = p.r.choice(able)
    return parents


@pytest.mark.parametrize("seqs,longest,page,family,empty", [
    (1, 50, 16, 1, 0), (2, 100, 16, 1, 0.5), (64, 300, 16, 1, 0.7), (300, 40, 16, 4, 0.6), (1030, 60, 3, 2, 0.5),
    (2500, 10, 1, 3, 0.8), (40, 9000, 16, 1, 0.7), (70, 0, 16, 1, 1.0), (5000, 33, 32, 1, 0.9)])
def test_forks(seqs, longest, page, family, empty):
    p = Pool(seqs + page, seqs, longest, page, family, spare=seqs + 3, empty=empty)
    if seqs == 2:
        p.lens[0] = 0
    parents = children(p)
    assert_fork(run_fork(p, parents), fork_reference(p, parents))


@pytest.mark.parametrize("room", [0, 1, 5, 40])
@pytest.mark.parametrize("seqs", [100, 3000])
def test_forks_with_too_few_pages(room, seqs):
    p = Pool(room, seqs, 90, 16, empty=0.6, spare=room)
    parents = children(p)
    want = fork_reference(p, parents)
    assert room >= 40 or tl.TOPLOC_SEQ_NO_PAGES in want[7]
    assert_fork(run_fork(p, parents), want)
    assert_fork(run_fork(p, parents, head=-3), fork_reference(p, parents, head=-3))
    past = len(p.free) + 2
    assert_fork(run_fork(p, parents, head=past), fork_reference(p, parents, head=past))


def test_forks_that_are_refused():
    p = Pool(5, 60, 200, 16, empty=0.6, spare=70)
    parents = children(p, 0.9)
    able, no = np.nonzero(p.lens > 32)[0], np.nonzero(parents >= 0)[0]
    parents[no[0]] = 60                                # no such sequence
    parents[no[1]] = 2 ** 31 - 1
    parents[no[2]] = no[3]                             # a child itself
    parents[no[4]] = no[4]
    parents[no[5]] = able[0]
    p.table[able[0], 1] = p.pages                      # outside the pool
    parents[no[6]] = able[1]
    p.table[able[1], 0] = -1
    parents[able[2]] = able[3]                         # holds tokens
    parents[no[7]] = able[4]
    p.lens[able[4]] = p.width * 16 + 1                 # more than a row
    parents[no[8]] = able[5]
    p.lens[able[5]] = -4
    want = fork_reference(p, parents)
    assert {tl.TOPLOC_SEQ_BAD_PARENT, tl.TOPLOC_SEQ_IN_USE, tl.TOPLOC_SEQ_BAD_PAGE, tl.TOPLOC_SEQ_BAD_LENGTH} <= set(want[7])
    assert_fork(run_fork(p, parents), want)
    free = p.free.copy()
    free[p.head + 1] = p.pages                         # the list names a page that does not exist
    assert_fork(run_fork(p, parents, free=free), fork_reference(p, parents, free=free))


# ---- releases --------------------------------------------------------------------------------------

def release_reference(p, gone, head=None, num_free=None):
    free = p.free[:num_free].copy()
    head = p.head if head is None else head
    room = min(max(head, 0), len(free))
    left, kv, status = p.shares.astype(np.int64), p.lens.copy(), np.zeros(p.n)
    held = np.zeros(p.n, bool)
    for i in np.nonzero(gone)[0]:
        have = pages_of(max(int(p.lens[i]), 0), p.page)
        if p.lens[i] < 0 or have > p.width:
            status[i] = tl.TOPLOC_SEQ_BAD_LENGTH
        row = p.table[i, :min(have, p.width)]
        held[i] = len(row) > 0
        good = (row >= 0) & (row < p.pages)
        if not good.all():
            status[i] = tl.TOPLOC_SEQ_BAD_PAGE
        np.subtract.at(left, row[good], 1)
        kv[i] = 0
    back = np.nonzero(left < 0)[0]
    fit = min(len(back), room)
    free[room - fit:room] = back[:fit]
    if len(back) > room:
        status[gone.astype(bool) & held & (status == 0)] = tl.TOPLOC_SEQ_NO_ROOM
    return free, kv, np.maximum(left, 0), room - fit, status


def run_release(p, gone, head=None, num_free=None, repeat=2):
    free = ints(p.free[:num_free])
    out = [ints(np.full(s, -9)) for s in (p.n, p.pages, 1)] + [ints(np.full(p.n, 99), torch.uint8)]
    args = [ints(gone, torch.uint8), ints(p.lens), ints(p.table), ints(p.shares), p.page, free,
            ints([p.head if head is None else head])]
    for _ in range(repeat):
        tl.toploc_release_pages(*args, *out)
    torch.cuda.synchronize()
    return [host(t) for t in [free] + out]


def assert_release(got, want):
    free, kv, shares, following, status = want
    assert np.array_equal(got[0], free) and np.array_equal(got[1], kv) and np.array_equal(got[2], shares)
    assert got[3].tolist() == [following] and got[4].tolist() == status.tolist()


@pytest.mark.parametrize("seqs,longest,page,family,share", [
    (1, 50, 16, 1, 1.0), (64, 2048, 16, 1, 0.3), (64, 300, 16, 8, 1.0), (300, 100, 7, 4, 0.5), (1030, 60, 3, 2, 0.5),
    (40, 20000, 16, 5, 0.7), (3000, 200, 1, 1, 0.0), (9000, 3, 1, 3, 0.5)])
def test_releases(seqs, longest, page, family, share):
    p = Pool(seqs + page, seqs, longest, page, family)
    gone = (p.r.random(seqs) < share) * p.r.integers(1, 256, seqs)
    assert_release(run_release(p, gone), release_reference(p, gone))


def test_releases_of_what_is_not_as_promised():
    p = Pool(3, 50, 200, 16)
    gone = np.ones(50, np.int64)
    able = np.nonzero(p.lens > 40)[0]
    p.table[able[0], 1] = p.pages
    p.table[able[1], 0] = -1
    p.table[able[2], 1] = p.table[able[2], 0]          # a page twice: it comes back once
    p.lens[able[3]] = -1
    p.lens[able[4]] = 2 ** 31 - 1
    p.table[able[4]] = np.clip(p.table[able[4]], 0, p.pages - 1)
    assert_release(run_release(p, gone), release_reference(p, gone))


@pytest.mark.parametrize("head", [-5, 0, 3, 10 ** 6])
def test_a_free_list_without_room(head):
    p = Pool(4, 50, 200, 16)
    gone = (p.r.random(50) < 0.8).astype(np.int64)
    for num_free in (None, 5):
        want = release_reference(p, gone, head, num_free)
        assert_release(run_release(p, gone, head, num_free), want)
        assert head == 10 ** 6 and num_free is None or tl.TOPLOC_SEQ_NO_ROOM in want[4]


# ---- compaction ------------------------------------------------------------------------------------

def compact_reference(p, extra=0):
    held, status = [], np.zeros(p.n)
    for i in range(p.n):
        have = pages_of(max(int(p.lens[i]), 0), p.page)
        if p.lens[i] < 0 or have > p.width:
            status[i] = tl.TOPLOC_SEQ_BAD_LENGTH
        row = p.table[i, :min(have, p.width)]
        held.append(row)
        if ((row < 0) | (row >= p.pages)).any():
            status[i] = tl.TOPLOC_SEQ_BAD_PAGE
    live = np.zeros(p.pages, bool)
    for row in held:
        live[row[(row >= 0) & (row < p.pages)]] = True
    n = int(live.sum())
    source, target = np.nonzero(live[n:])[0] + n, np.nonzero(~live[:n])[0]
    moved = np.arange(p.pages)
    moved[source] = target
    table = np.full_like(p.table, -7)
    for i, row in enumerate(held):
        good = (row >= 0) & (row < p.pages)
        table[i, :len(row)] = np.where(good, moved[np.where(good, row, 0)] if p.pages else 0, row)
    shares = np.zeros_like(p.shares)
    shares[moved[live]] = p.shares[live]
    free = np.full(p.pages + extra, -9)
    free[n + extra:] = np.arange(n, p.pages)
    fill = np.full(p.pages - len(source), -1)
    return (table, shares, free, np.concatenate([source, fill]), np.concatenate([target, fill]), len(source), n + extra,
            status)


def run_compact(p, extra=0, in_place=False, repeat=2):
    table_in = ints(p.table)
    table = table_in if in_place else ints(np.full_like(p.table, -7))
    out = [table] + [ints(np.full(s, -9)) for s in (p.pages, p.pages + extra, p.pages, p.pages, 1, 1)]
    out += [ints(np.full(p.n, 99), torch.uint8)]
    for _ in range(1 if in_place else repeat):
        tl.toploc_compact_pages(ints(p.lens), table_in, ints(p.shares), p.page, *out)
    torch.cuda.synchronize()
    return [host(t) for t in out]


def assert_compact(got, want, in_place=None):
    assert got[7].tolist() == want[7].tolist()
    table = want[0] if in_place is None else np.where(want[0] == -7, in_place, want[0])
    assert np.array_equal(got[0], table)
    for g, w in zip(got[1:5], want[1:5]):
        assert np.array_equal(g, w)
    assert got[5].tolist() == [want[5]] and got[6].tolist() == [want[6]]


@pytest.mark.parametrize("seqs,longest,page,family,spare", [
    (1, 50, 16, 1, 20), (1, 50, 16, 1, 0), (64, 2048, 16, 1, 3000), (64, 300, 16, 8, 5), (300, 100, 7, 4, 500),
    (1030, 60, 3, 2, 20000), (40, 20000, 16, 5, 100), (9000, 3, 1, 3, 1), (20, 0, 16, 1, 40)])
def test_compaction(seqs, longest, page, family, spare):
    p = Pool(seqs + page, seqs, longest, page, family, spare)
    want = compact_reference(p)
    assert_compact(run_compact(p), want)
    assert_compact(run_compact(p, in_place=True), want, p.table)
    assert_compact(run_compact(p, extra=7), compact_reference(p, extra=7))


def test_compaction_with_entries_that_are_not_as_promised():
    p = Pool(6, 50, 200, 16, spare=90)
    able = np.nonzero(p.lens > 40)[0]
    p.table[able[0], 1] = p.pages
    p.table[able[1], 0] = -1
    p.lens[able[2]] = -1
    p.lens[able[3]] = 2 ** 31 - 1
    assert_compact(run_compact(p), compact_reference(p))


def test_an_empty_pool():
    p = Pool(7, 4, 0, 16, spare=0)
    assert p.pages == 0
    assert_compact(run_compact(p), compact_reference(p))
    assert_release(run_release(p, np.ones(4)), release_reference(p, np.ones(4)))
    parents = np.array([-1, 0, 0, 7])
    assert_fork(run_fork(p, parents), fork_reference(p, parents))
    none = Pool(8, 0, 5, 16, spare=9)
    assert_compact(run_compact(none), compact_reference(none))
    assert_release(run_release(none, np.zeros(0)), release_reference(none, np.zeros(0)))
    assert_fork(run_fork(none, np.zeros(0)), fork_reference(none, np.zeros(0)))


def test_tables_in_a_wider_one():
    """Rows further apart than they are long; compaction into the columns beside them."""
    p = Pool(9, 30, 100, 16, spare=40)
    wide = ints(np.full((30, 2 * p.width + 3), -7))
    here, there = wide[:, :p.width], wide[:, p.width + 2:2 * p.width + 2]
    here.copy_(ints(p.table))
    want = compact_reference(p)
    out = [ints(np.full(s, -9)) for s in (p.pages, p.pages, p.pages, p.pages, 1, 1)] + [ints(np.zeros(30), torch.uint8)]
    tl.toploc_compact_pages(ints(p.lens), here, ints(p.shares), 16, there, *out)
    assert np.array_equal(host(there), want[0]) and np.array_equal(host(here), p.table)
    assert (host(wide[:, p.width:p.width + 2]) == -7).all()
    with pytest.raises(tl.ToplocError):                # shifted by one column: the tables meet
        tl.toploc_compact_pages(ints(p.lens), here, ints(p.shares), 16, wide[:, 1:p.width + 1], *out)


# ---- copies ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,heads,dim,order,caches", [
    (16, 8, 128, "token", 4), (16, 2, 64, "head", 3), (1, 1, 1, "token", 2), (3, 5, 7, "token", 2), (7, 3, 9, "head", 1),
    (128, 8, 128, "token", 2), (16, 2, 64, "apart", 2), (5, 3, 7, "apart", 2), (5, 3, 6, "apart", 1), (16, 1, 64, "token", 150)])
def test_copies(dtype, page, heads, dim, order, caches):
    g = torch.Generator(device=DEV)
    g.manual_seed(page * dim)
    pages = 40
    store = torch.randn((caches, pages) + ((page, heads) if order != "head" else (heads, page)) + (dim,), generator=g,
                        device=DEV).to(dtype)
    if order == "head":
        views = [c.transpose(1, 2) for c in store]
    elif order == "apart":                             # every head's row padded, so that a page is no run
        store = torch.randn((caches, pages, page, heads, dim + 2 + dim % 2), generator=g, device=DEV).to(dtype)
        views = [c[..., :dim] for c in store]
    else:
        views = list(store)
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    source, target = perm[:15].clone(), perm[15:30].clone()
    source[3], target[5], target[6] = -1, pages, 2 ** 31 - 1   # skipped
    want = store.clone()
    for i in range(13):
        s, t = int(source[i]), int(target[i])
        if i not in (3, 5, 6):
            (want[:, t, ..., :dim] if order == "apart" else want[:, t]).copy_(
                want[:, s, ..., :dim] if order == "apart" else want[:, s])
    tl.toploc_copy_pages(views, source, target, ints([13]))
    assert torch.equal(store, want)
    for count in (0, -1):
        tl.toploc_copy_pages(views, source, target, ints([count]))
    assert torch.equal(store, want)
    tl.toploc_copy_pages(views, source[:2], target[:2], ints([10 ** 6]))       # no more than the list holds
    assert torch.equal(store, want)


def test_copies_of_pages_past_32_bits():
    """The last pages of a cache of 2^33 bytes."""
    cache = torch.empty((1 << 13, 64, 64, 128), dtype=torch.bfloat16, device=DEV)
    cache[-2] = 3.0
    cache[-1] = 5.0
    cache[0] = 7.0
    last = (1 << 13) - 1
    tl.toploc_copy_pages([cache], ints([last - 1, last]), ints([last - 2, 0]), ints([2]))
    assert cache[-3].eq(3).all() and cache[0].eq(5).all() and cache[-1].eq(5).all()


# ---- together --------------------------------------------------------------------------------------

def test_plan_fork_release_and_compact_together():
    """A pool over many steps: prompts are planned, forked, decoded, released, compacted.  After each step no page has two
    uses and none is lost, and every sequence still reads its own tokens."""
    r = np.random.default_rng(11)
    n, page, width, pages, heads, dim = 24, 4, 20, 240, 2, 8
    caches = [torch.zeros((pages, page, heads, dim), dtype=torch.float32, device=DEV) for _ in range(2)]
    table, free = ints(np.full((n, width), -1)), ints(r.permutation(pages))
    lens, shares, head = ints(np.zeros(n)), ints(np.zeros(pages)), ints([0])
    status = ints(np.zeros(n), torch.uint8)
    text = [[] for _ in range(n)]                      # what each sequence holds: one number a token
    number = 0

    def check():
        assert not status.any(), status
        have, rows, t = host(lens), host(table), [host(c) for c in caches]
        used = np.zeros(pages, int)
        for i in range(n):
            assert have[i] == len(text[i])
            row = rows[i, :pages_of(int(have[i]), page)]
            used[row] += 1
            for pos, want in enumerate(text[i]):
                assert (t[0][row[pos // page], pos % page] == want).all() and (t[1][row[pos // page], pos % page] == -want).all()
        assert np.array_equal(host(shares), np.maximum(used - 1, 0))
        rest = host(free)[int(head):]
        assert len(set(rest)) == len(rest) == pages - (used > 0).sum() and not used[rest].any()

    for step in range(40):
        kind = step % 5
        out_lens, out_shares, following = torch.empty_like(lens), torch.empty_like(shares), torch.empty_like(head)
        source, target, copies = torch.empty_like(lens), torch.empty_like(lens), torch.empty_like(head)
        if kind in (0, 2, 3):                          # new tokens for sequences that have some, or prompts
            new = [int(r.integers(1, 12)) if kind == 0 and not text[i] and r.random() < 0.3 else
                   int(r.integers(0, 3)) if text[i] and len(text[i]) < 40 else 0 for i in range(n)]
            tokens = sum(new)
            offsets = torch.empty(n + 1, dtype=torch.int32, device=DEV)
            slots, positions = torch.empty(tokens, dtype=torch.int64, device=DEV), torch.empty(tokens, dtype=torch.int32, device=DEV)
            tl.toploc_plan_pages(lens, ints(new), free, head, table, page, offsets, out_lens, slots, positions, following,
                                 status)
            numbers = np.arange(number, number + tokens) + 1.0
            number += tokens
            k = ints(numbers, torch.float32)[:, None, None].expand(tokens, heads, dim).contiguous()
            tl.toploc_cache_write(k, -k, slots, *caches)
            at = 0
            for i in range(n):
                text[i] += list(numbers[at:at + new[i]])
                at += new[i]
        elif kind == 1:                                # samples of what is there
            able = [i for i in range(n) if text[i]]
            parents = [int(r.choice(able)) if able and not text[i] and r.random() < 0.5 else -1 for i in range(n)]
            tl.toploc_fork_pages(ints(parents), lens, shares, free, head, table, page, out_lens, out_shares, source, target,
                                 copies, following, status)
            tl.toploc_copy_pages(caches, source, target, copies)
            text = [list(text[parents[i]]) if parents[i] >= 0 else text[i] for i in range(n)]
            shares = out_shares
        else:
            gone = [int(bool(text[i]) and r.random() < 0.5) for i in range(n)]
            tl.toploc_release_pages(ints(gone, torch.uint8), lens, table, shares, page, free, head, out_lens, out_shares,
                                    following, status)
            text = [[] if gone[i] else text[i] for i in range(n)]
            shares = out_shares
        lens, head = out_lens, following
        check()
        if step % 10 == 9:
            out_shares, following = torch.empty_like(shares), torch.empty_like(head)
            source, target = ints(np.zeros(pages)), ints(np.zeros(pages))
            tl.toploc_compact_pages(lens, table, shares, page, table, out_shares, free, source, target, copies, following,
                                    status)
            tl.toploc_copy_pages(caches, source, target, copies)
            shares, head = out_shares, following
            check()
            assert int(head) == len({p for i in range(n) for p in host(table)[i, :pages_of(len(text[i]), page)]})


def test_captured_and_replayed_on_another_stream():
    p = Pool(12, 64, 300, 16, empty=0.7, spare=80)
    parents = children(p)
    want = fork_reference(p, parents)
    cache = torch.randn((p.pages, 16, 2, 64), device=DEV)
    begun = cache.clone()
    table = ints(p.table)
    out = [ints(np.full(s, -9)) for s in (p.n, p.pages, p.n, p.n, 1, 1)] + [ints(np.full(p.n, 99), torch.uint8)]
    args = [ints(parents), ints(p.lens), ints(p.shares), ints(p.free), ints([p.head]), table, p.page]
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        tl.toploc_fork_pages(*args, *out)
        tl.toploc_copy_pages([cache], out[2], out[3], out[4])
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert_fork([host(t) for t in [table] + out], want)
    k = want[5]
    assert torch.equal(cache[ints(want[4][:k], torch.int64)], begun[ints(want[3][:k], torch.int64)])


@pytest.mark.parametrize("seqs,longest,page,family,spare", [
    (2500, 1500, 16, 3, 10),       # a release of many pages: three launches
    (5, 100, 16, 1, 300000),       # few pages of a large pool are held: a warp's range is longer than its lanes' marks
    (600, 3000, 8, 2, 280000)])
def test_large_pools(seqs, longest, page, family, spare):
    p = Pool(seqs, seqs, longest, page, family, spare, empty=0.3)
    gone = (p.r.random(seqs) < 0.6).astype(np.int64)
    assert_release(run_release(p, gone), release_reference(p, gone))
    assert_compact(run_compact(p), compact_reference(p))
    parents = children(p)
    assert_fork(run_fork(p, parents), fork_reference(p, parents))


def test_large_releases_of_what_is_not_as_promised():
    p = Pool(13, 2500, 1500, 16, 3)
    gone = np.ones(2500, np.int64)
    able = np.nonzero(p.lens > 700)[0]
    p.table[able[0], 1] = p.pages
    p.table[able[1], 0] = -1
    p.table[able[2], 1] = p.table[able[2], 0]
    p.lens[able[3]] = -1
    p.lens[able[4]] = 2 ** 31 - 1
    p.table[able[4]] = np.clip(p.table[able[4]], 0, p.pages - 1)
    assert_release(run_release(p, gone), release_reference(p, gone))
    for head in (-5, 0, 1000, 10 ** 6):
        want = release_reference(p, gone, head)
        assert_release(run_release(p, gone, head), want)
        assert head == 10 ** 6 or tl.TOPLOC_SEQ_NO_ROOM in want[4]


def test_forks_among_a_hundred_thousand_sequences():
    """Many sequences a thread of the plan."""
    p = Pool(14, 100000, 20, 16, empty=0.5, spare=30000)
    parents = children(p)
    want = fork_reference(p, parents)
    assert tl.TOPLOC_SEQ_NO_PAGES in want[7]
    assert_fork(run_fork(p, parents), want)
