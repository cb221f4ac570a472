"""Forks with their copies, and releases and compactions of shared pages, on other streams, several at once, in graphs."""
import threading

import numpy as np
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(values, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(values)).to(device=DEV, dtype=dtype)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def calls(seed, parents, children, longest, page=4):
    """A fork with its copies; a release of half of what it left; a compaction of that with its copies.  Functions of a stream
    that return what they wrote."""
    r = np.random.default_rng(seed)
    n, each = parents * (children + 1), children + 1
    lens = np.zeros(n, np.int64)
    lens[::each] = r.integers(1, longest + 1, parents)
    have = -(-lens // page)
    pages, width = 2 * int(have.sum()) + n, int(have.max()) + 2
    perm = r.permutation(pages)
    table = np.full((n, width), -1)
    table[np.arange(width)[None, :] < have[:, None]] = perm[:have.sum()]
    parent = np.where(np.arange(n) % each == 0, -1, np.arange(n) // each * each)
    parent[(np.arange(n) % each != 0) & (r.random(n) < 0.2)] = -1
    parent, lens, table, free, head = ints(parent), ints(lens), ints(table), ints(perm), ints([int(have.sum())])
    shares, gone = ints(np.zeros(pages)), ints(r.integers(0, 2, n), torch.uint8)
    cache = torch.randn((pages, page, 2, 16), device=DEV)

    def fork(stream):
        rows, moved = table.clone(), cache.clone()
        out = [torch.empty_like(t) for t in (lens, shares, lens, lens, head, head, gone)]
        torch.cuda.current_stream().synchronize()
        tl.toploc_fork_pages(parent, lens, shares, free, head, rows, page, *out, stream=stream)
        tl.toploc_copy_pages([moved], out[2], out[3], out[4], stream=stream)
        return [rows] + out + [moved]

    forked = fork(None)
    torch.cuda.synchronize()
    rows, kv_lens, held, _, _, _, taken, status, filled = forked
    assert not status.any() and int(held.max()) > 0 and int(taken) > int(head)

    def release(stream):
        back = free.clone()
        out = [torch.empty_like(t) for t in (lens, shares, head, gone)]
        torch.cuda.current_stream().synchronize()
        tl.toploc_release_pages(gone, kv_lens, rows, held, page, back, taken, *out, stream=stream)
        return [back] + out

    def compact(stream):
        out, moved = [rows.clone(), torch.empty_like(shares), free.clone()], filled.clone()
        out += [torch.empty_like(t) for t in (shares, shares, head, head, gone)]
        torch.cuda.current_stream().synchronize()
        tl.toploc_compact_pages(kv_lens, rows, held, page, *out, stream=stream)
        tl.toploc_copy_pages([moved], out[3], out[4], out[5], stream=stream)
        return out + [moved]

    return fork, release, compact


SIZES = [(3, 4, 60), (64, 7, 300), (90, 9, 900)]       # one block; a cluster; releases in three launches


def test_sizes_are_of_all_kinds():
    """Entries and pages, which the planners choose by."""
    work = []
    for i, size in enumerate(SIZES):
        rows, pages = (f(None) for f in calls(i, *size)[:2])
        work.append(rows[0].numel() + pages[0].numel())
    assert work[0] <= 8192 < work[1] <= 131072 < work[2]


@pytest.mark.parametrize("size", SIZES)
def test_contents_follow_the_table(size):
    """Through a fork every child reads its parent's tokens; through a compaction every sequence its own."""
    fork, _, compact = calls(10, *size)
    rows, lens, _, _, _, _, _, _, cache = fork(None)
    moved = compact(None)
    torch.cuda.synchronize()
    each, page = size[1] + 1, cache.shape[1]
    lens = lens.tolist()

    def tokens(cache, table, i):
        return cache[table[i, :-(-lens[i] // page)].long()].flatten(0, 1)[:lens[i]]

    for i in range(0, len(lens), max(1, len(lens) // 97)):
        first = i // each * each
        assert lens[i] in (0, lens[first])
        assert torch.equal(tokens(cache, rows, i), tokens(cache, rows, first)[:lens[i]])
        assert torch.equal(tokens(moved[-1], moved[0], i), tokens(cache, rows, i))


@pytest.mark.parametrize("size", SIZES)
def test_on_a_stream_of_its_own(size):
    side = torch.cuda.Stream()
    for call in calls(1, *size):
        want = call(None)
        torch.cuda.synchronize()
        got = call(side)
        side.synchronize()
        assert same(got, want), call.__name__


@pytest.mark.parametrize("size", SIZES)
def test_two_calls_at_once(size):
    streams = [torch.cuda.Stream() for _ in range(2)]
    for a, b in zip(calls(2, *size), calls(3, *size)):
        want = [a(None), b(None)]
        torch.cuda.synchronize()
        for _ in range(5):
            got = [a(streams[0]), b(streams[1])]
            torch.cuda.synchronize()
            assert same(got[0], want[0]) and same(got[1], want[1]), a.__name__


def test_from_several_threads():
    all_calls = [calls(seed, *SIZES[seed % 3]) for seed in range(4)]
    want = [[call(None) for call in some] for some in all_calls]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        for _ in range(5):
            for call, expected in zip(all_calls[i], want[i]):
                with torch.cuda.stream(stream):
                    got = call(stream)
                stream.synchronize()
                if not same(got, expected):
                    wrong.append(call.__name__)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@pytest.mark.parametrize("size", SIZES)
def test_one_graph_of_a_samples_life(size):
    """Fork, copies, release and compaction as one graph on a side stream, replayed."""
    parents, children, longest = size
    fork, _, _ = calls(20, *size)
    rows, kv_lens, held, _, _, _, taken, status, cache = fork(None)
    torch.cuda.synchronize()
    n, pages, page = len(kv_lens), cache.shape[0], cache.shape[1]
    gone = ints(np.arange(n) % 3 == 0, torch.uint8)
    back = torch.arange(pages, dtype=torch.int32, device=DEV)
    ended = [torch.empty_like(t) for t in (kv_lens, held, taken, status)]
    out = [torch.empty_like(t) for t in (rows, held, back, held, held, taken, taken, status)]
    begun = cache.clone()

    def steps():
        cache.copy_(begun)
        tl.toploc_release_pages(gone, kv_lens, rows, held, page, back, taken, *ended)
        tl.toploc_compact_pages(ended[0], rows, ended[1], page, *out)
        tl.toploc_copy_pages([cache], out[3], out[4], out[5])

    for t in out:
        t.zero_()
    steps()
    torch.cuda.synchronize()
    written = ended + out + [back, cache]
    want = [t.clone() for t in written]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        steps()
    for _ in range(3):
        for t in ended + out[1:2] + out[3:]:
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert same(written, want)
