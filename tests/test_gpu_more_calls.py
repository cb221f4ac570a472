"""Norm with rotation, log probabilities and pools: other streams, several calls at once, tensors past 32 bits."""
import threading

import numpy as np
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def calls(seed):
    """One call of each operator on inputs of this seed: functions of a stream that return what it wrote."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV).bfloat16()

    q, k, freq = normal(700, 8, 128), normal(700, 2, 128), torch.rand(64, generator=g, device=DEV)
    positions = torch.arange(700, device=DEV, dtype=torch.int32) * 31
    slots = torch.randperm(64 * 16, generator=g, device=DEV)[:700]
    x = normal(40, 50001) * 3
    tokens = torch.randint(50001, (40,), generator=g, device=DEV)
    r = np.random.default_rng(seed)
    n, pages, page = 200, 6000, 4
    lens = r.integers(0, 90, n)
    have = -(-lens // page)
    table = np.full((n, 30), -1)
    table[np.arange(30)[None, :] < have[:, None]] = r.permutation(pages)[:have.sum()]
    held = int(have.sum())
    gone = r.integers(0, 2, n)
    lens_t, table_t = ints(lens.tolist()), torch.from_numpy(table).to(DEV, torch.int32)
    gone_t, shares, head = ints(gone.tolist(), torch.uint8), ints([0] * pages), ints([held])
    free = torch.from_numpy(r.permutation(pages)).to(DEV, torch.int32)
    cache = normal(pages, page, 2, 64)

    def prompt(stream):
        return tl.toploc_norm_rotary_prompt(q, k, positions, freq, stream=stream)

    def paged(stream):
        caches = [normal(64, 16, 2, 128).zero_() for _ in range(2)]
        torch.cuda.current_stream().synchronize()
        return [tl.toploc_norm_rotary_paged(q, k, k, positions, slots, freq, *caches, stream=stream)] + caches

    def logprobs(stream):
        return tl.toploc_token_logprobs(x, tokens, 7, want_entropy=True, stream=stream)

    def release(stream):
        out = [torch.empty_like(lens_t), torch.empty_like(shares), torch.empty_like(head), torch.empty_like(gone_t)]
        back = free.clone()
        torch.cuda.current_stream().synchronize()
        tl.toploc_release_pages(gone_t, lens_t, table_t, shares, page, back, head, *out, stream=stream)
        return [back] + out

    def compact(stream):
        # (the front of the free list is left as it is)
        out = [table_t.clone(), torch.empty_like(shares), free.clone()]
        out += [torch.empty_like(t) for t in (free, free, head, head, gone_t)]
        moved = cache.clone()
        torch.cuda.current_stream().synchronize()
        tl.toploc_compact_pages(lens_t, table_t, shares, page, *out, stream=stream)
        tl.toploc_copy_pages([moved], out[3], out[4], out[5], stream=stream)
        return out + [moved]

    return prompt, paged, logprobs, release, compact


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_on_a_stream_of_its_own():
    side = torch.cuda.Stream()
    for call in calls(1):
        want = call(None)
        torch.cuda.synchronize()
        got = call(side)
        side.synchronize()
        assert same(got, want), call.__name__


def test_two_calls_at_once():
    """Calls of different inputs on two streams: nothing is shared between them."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [calls(2), calls(3)]
    for a, b in zip(*both):
        want = [a(None), b(None)]
        torch.cuda.synchronize()
        for _ in range(5):
            got = [a(streams[0]), b(streams[1])]
            torch.cuda.synchronize()
            assert same(got[0], want[0]) and same(got[1], want[1]), a.__name__


def test_from_several_threads():
    all_calls = [calls(seed) for seed in range(4, 8)]
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


def test_one_graph_of_all_replayed():
    side = torch.cuda.Stream()
    q, k = torch.randn((64, 4, 64), device=DEV), torch.randn((64, 2, 64), device=DEV)
    positions, freq = torch.arange(64, device=DEV, dtype=torch.int32), torch.rand(32, device=DEV)
    x = torch.randn((3, 3000), device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = list(tl.toploc_norm_rotary_prompt(q, k, positions, freq)) + list(tl.toploc_token_logprobs(x, top=4)[2:])
    for _ in range(2):
        q.normal_()
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = list(tl.toploc_norm_rotary_prompt(q, k, positions, freq)) + list(tl.toploc_token_logprobs(x, top=4)[2:])
        assert same(got, want)


def test_rotary_in_a_cache_past_32_bits():
    """The last page of a cache of 2^32 elements, keys and values in one tensor."""
    cache = torch.empty((1 << 13, 64, 64, 128), dtype=torch.bfloat16, device=DEV)
    cache[-1] = 0
    k_cache, v_cache = cache[:, :, :32], cache[:, :, 32:]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v = (torch.randn((3, 32, 128), generator=g, device=DEV).bfloat16() for _ in range(3))
    positions = ints([5, 6, 7])
    freq = torch.rand(64, generator=g, device=DEV)
    last = (1 << 13) * 64
    slots = ints([last - 1, last, last - 64], torch.int64)
    tl.toploc_norm_rotary_paged(q, k, v, positions, slots, freq, k_cache, v_cache)
    want = tl.toploc_norm_rotary_prompt(q, k, positions, freq)[1]
    assert torch.equal(k_cache[-1, 63], want[0]) and torch.equal(k_cache[-1, 0], want[2])
    assert torch.equal(v_cache[-1, 63], v[0]) and torch.equal(v_cache[-1, 0], v[2])
    assert not cache[-1, 1:63].any()


def test_rotary_of_heads_far_apart():
    """Heads 2^26 elements from each other: more than the 32-bit places of the kernel on vectors reach."""
    flat = torch.empty((1 << 27) + (1 << 10), dtype=torch.bfloat16, device=DEV)
    q = flat.as_strided((4, 3, 128), (128, 1 << 26, 1))
    q.copy_(torch.randn((4, 3, 128), device=DEV))
    k = torch.randn((4, 1, 128), device=DEV).bfloat16()
    positions, freq = ints([0, 9, 100, 5000]), torch.rand(64, device=DEV)
    want = tl.toploc_norm_rotary_prompt(q.contiguous(), k, positions, freq)
    got = tl.toploc_norm_rotary_prompt(q, k, positions, freq)
    assert torch.allclose(got[0].float(), want[0].float(), rtol=2 ** -7, atol=2 ** -20) and torch.equal(got[1], want[1])


def test_logits_past_32_bits():
    """Rows that begin behind 2^32 bytes and 2^31 elements."""
    x = torch.zeros((17000, 128000), dtype=torch.bfloat16, device=DEV)
    x[-1] = torch.randn(128000, device=DEV)
    x[-2, 127999] = 20.0
    tokens = torch.full((17000,), 127999, device=DEV)
    got = tl.toploc_token_logprobs(x, tokens, 3, want_entropy=True)
    want = tl.toploc_token_logprobs(x[-2:].clone(), tokens[-2:], 3, want_entropy=True)
    assert torch.equal(got[2][-2:], want[2]) and got[2][-2, 0].item() == 127999
    for a, b in zip(got, want):
        assert torch.allclose(a[-2:].double(), b.double(), rtol=0, atol=1e-5)
    assert (got[2][:-2] == ints([0, 1, 2], torch.int64)).all()
    log = float(np.log(128000))
    # 2^-24 (62 sums of partial sums in a row and 45 more) of a sum, and roundings of 12
    assert (got[0][:-2] + log).abs().max().item() < 1e-5 and (got[1][:-2] - log).abs().max().item() < 2e-5


@pytest.mark.parametrize("before", ["nothing", "set", "copy", "kernel", "another stream", "two streams"])
def test_copies_captured_behind_anything(before):
    """The copies may begin before a kernel in front of them has ended; what is in front may be something else."""
    cache = torch.randn((8, 16, 2, 64), device=DEV)
    begun = cache.clone()
    source, target, count = ints([0, 0, 0]), ints([4, 5, 6]), ints([3])
    pages, other = ints([1, 2, 3]), torch.zeros(1 << 22, device=DEV)
    side, third = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        if before == "set":
            other.zero_()
            source.zero_()
        elif before == "copy":
            source.copy_(pages)
        elif before == "kernel":
            source.add_(1)
        elif before != "nothing":
            third.wait_stream(side)
            with torch.cuda.stream(third):
                other.add_(1)
                source.copy_(pages)
            if before == "two streams":
                count.add_(0)
            side.wait_stream(third)
        tl.toploc_copy_pages([cache], source, target, count)
    graph.replay()
    torch.cuda.synchronize()
    first = {"nothing": [0, 0, 0], "set": [0, 0, 0], "kernel": [1, 1, 1]}.get(before, [1, 2, 3])
    assert torch.equal(cache[4:7], begun[first])
    assert torch.equal(cache[:4], begun[:4]) and torch.equal(cache[7], begun[7])
