"""Outputs of norm and rotation in the memory of other arguments: refused before any CUDA call, compared with sets of bytes.
No kernel is launched here."""
import ctypes
import random

import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would run on made-up addresses")
INVALID, UNSUPPORTED = -1, -2
BASE = 1 << 24


@pytest.fixture(scope="module")
def lib():
    from paper_2501_16007_b200.csrc import build
    build.build()
    from paper_2501_16007_b200 import model_ops
    return model_ops._library()


def layout(q_heads, kv_heads, tokens, dim, strides, size, turned=2):
    names = ("q", "k", "v", "q_out", "k_out")
    s = {}
    for name in names:
        s[name + "_token_stride"], s[name + "_head_stride"] = strides.get(name, (1 << 12, dim))
    return tl.ToplocRotaryLayout(dtype=1 if size == 4 else 0, head_dim=dim, q_heads=q_heads, kv_heads=kv_heads,
                                 rotary_dim=turned, pairing=0, num_tokens=tokens, eps=0.0, reserved=0, **s)


def at(offset):
    return ctypes.c_void_p(BASE + offset)


FAR = {name: (i + 1) << 22 for i, name in enumerate(("q", "k", "v", "pos", "freq", "qw", "kw", "slots", "q_out", "k_out", "kc",
                                                     "vc"))}


def prompt(lib, lay, **places):
    a = {**FAR, **places}
    return lib.toploc_norm_rotary_prompt(at(a["q"]), at(a["k"]), at(a["pos"]), at(a["freq"]), at(a["qw"]), at(a["kw"]),
                                         ctypes.byref(lay), at(a["q_out"]), at(a["k_out"]), None)


def paged(lib, lay, **places):
    a = {**FAR, **places}
    kv = tl.ToplocKvLayout(page_size=16, num_pages=8, max_pages=0, reserved=0, table_stride=0, k_page_stride=1 << 14,
                           k_token_stride=1 << 10, k_head_stride=64, v_page_stride=1 << 14, v_token_stride=1 << 10,
                           v_head_stride=64)
    return lib.toploc_norm_rotary_paged(at(a["q"]), at(a["k"]), at(a["v"]), at(a["pos"]), at(a["slots"]), at(a["freq"]),
                                        at(a["qw"]), at(a["kw"]), ctypes.byref(lay), at(a["q_out"]), at(a["kc"]), at(a["vc"]),
                                        ctypes.byref(kv), None)


def taken(offset, heads, tokens, dim, strides, size):
    """Elements, as numbers of bytes."""
    return {offset + (t * strides[0] + h * strides[1] + c) * size for t in range(tokens) for h in range(heads)
            for c in range(dim)}


def passes(code):
    return code not in (0, INVALID, UNSUPPORTED)


@pytest.mark.parametrize("size", [2, 4])
def test_one_projection(lib, size):
    """Rows of queries, keys and values: in place, one head further on, into the keys, into the next row."""
    row, dim = 12 * 64, 64
    s = {n: (row, dim) for n in ("q", "k", "v", "q_out", "k_out")}
    lay = layout(8, 2, 5, dim, s, size)
    q, k, v, head = 0, 8 * dim * size, 10 * dim * size, dim * size
    for call in (prompt, paged):
        assert passes(call(lib, lay, q=q, k=k, v=v, q_out=q))
        assert passes(call(lib, lay, q=q, k=k, v=v))
        for wrong in (head, -head, size, k, v, k - 8 * head + size, row * size, row * size - head):
            assert call(lib, lay, q=1 << 16, k=(1 << 16) + k, v=(1 << 16) + v, q_out=(1 << 16) + wrong) == INVALID, wrong
    assert passes(prompt(lib, lay, q=q, k=k, q_out=q, k_out=k))
    assert passes(prompt(lib, lay, q=q, k=k, q_out=q, k_out=v))           # in the place of the values
    assert prompt(lib, lay, q=q, k=k, q_out=q, k_out=q) == INVALID
    # one head further on: the second head is read by another warp than the one that writes it
    assert prompt(lib, lay, q=q, k=k, q_out=q, k_out=k + head) == INVALID
    assert prompt(lib, lay, q=q, k=k, k_out=k - head) == INVALID


def test_rows_behind_the_last_one_are_free(lib):
    s = {n: (12 * 64, 64) for n in ("q", "k", "q_out", "k_out")}
    lay = layout(8, 2, 5, 64, s, 2)
    row = 12 * 64 * 2
    assert passes(prompt(lib, lay, q=0, k=1024, q_out=5 * row, k_out=5 * row + 1024))
    assert prompt(lib, lay, q=0, k=1024, q_out=4 * row, k_out=5 * row + 1024) == INVALID


def test_vectors(lib):
    lay = layout(4, 2, 100, 64, {}, 2, turned=64)
    for name, length in (("pos", 400), ("freq", 128), ("qw", 128), ("kw", 128)):
        for out in ("q_out", "k_out"):
            for call in (prompt, paged) if out == "q_out" else (prompt,):
                assert call(lib, lay, **{name: FAR[out] + 8}) == INVALID, (name, out)
                assert call(lib, lay, **{name: FAR[out] - length + 4}) == INVALID, (name, out)
                assert passes(call(lib, lay, **{name: FAR[out] - length})), (name, out)
                heads = 4 if out == "q_out" else 2
                assert passes(call(lib, lay, **{name: FAR[out] + heads * 128})), (name, out)   # between two rows
    assert paged(lib, lay, slots=FAR["q_out"] + (1 << 13)) == INVALID
    assert passes(paged(lib, lay, slots=FAR["q_out"] - 800))


@pytest.mark.parametrize("seed", range(8))
def test_against_sets_of_bytes(lib, seed):
    """Nothing is refused that shares no memory, and all is that does and has common steps or is in one piece."""
    r = random.Random(seed)
    seen = {True: 0, False: 0}
    for _ in range(3000):
        size, dim = r.choice((2, 4)), r.choice((2, 3, 4))
        q_heads, kv_heads, tokens = r.randint(1, 4), r.randint(1, 4), r.randint(1, 4)
        token, head = r.choice((0, dim, 4, 11, 16, 24, 40)), r.choice((dim, dim, 4, 5, 10, 32, 17))

        def steps():
            kind = r.random()
            if kind < 0.7:
                return token, head
            heads = max(q_heads, kv_heads)
            return (heads * dim, dim) if kind < 0.85 else (dim, tokens * dim)        # in one piece, either way

        s = {n: steps() for n in ("q", "k", "v", "q_out", "k_out")}
        places = {n: 4096 + 4 * r.randrange(100) for n in ("q", "k", "q_out", "k_out")}
        if r.random() < 0.2:
            places["q_out"], s["q_out"] = places["q"], s["q"]
        sets = {n: taken(places[n], q_heads if n[0] == "q" else kv_heads, tokens, dim, s[n], size) for n in places}
        share = lambda a, b: any(abs(x - y) < size for x in sets[a] for y in sets[b]) if size == 4 else bool(sets[a] & sets[b])
        in_place = places["q"] == places["q_out"], places["k"] == places["k_out"]
        pairs = [("q_out", "k"), ("k_out", "q"), ("q_out", "k_out")]
        pairs += [("q_out", "q")] * (not in_place[0]) + [("k_out", "k")] * (not in_place[1])
        if any(p and s[n] != s[n + "_out"] for p, n in zip(in_place, "qk")):
            continue                                   # (in place with other strides: refused as it always was)
        code = prompt(lib, layout(q_heads, kv_heads, tokens, dim, s, size), **places)
        shared = [p for p in pairs if share(*p)]
        seen[bool(shared)] += 1
        if not shared:
            assert passes(code), (s, places, q_heads, kv_heads, tokens, dim)
        elif any(s[a] == s[b] for a, b in shared):
            assert code == INVALID, (s, places, q_heads, kv_heads, tokens, dim)
    assert min(seen.values()) > 100, seen


def test_one_piece_in_the_gaps_of_another(lib):
    """An output in one piece, wherever it begins around rows with gaps."""
    tokens, heads, dim, row = 6, 2, 4, 20
    s = {"q": (row, dim), "q_out": (heads * dim, dim), "k": (64, dim), "k_out": (64, dim)}
    lay = layout(heads, heads, tokens, dim, s, 4)
    q = taken(4096, heads, tokens, dim, s["q"], 4)
    one = layout(heads, heads, 1, dim, s, 4)
    first = taken(4096, heads, 1, dim, s["q"], 4)
    for offset in range(4096 - 300, 4096 + 600, 4):
        if offset == 4096:
            continue
        out = taken(offset, heads, tokens, dim, s["q_out"], 4)
        assert (prompt(lib, lay, q=4096, q_out=offset) == INVALID) == bool(out & q), offset
        out = taken(offset, heads, 1, dim, s["q_out"], 4)
        assert (prompt(lib, one, q=4096, q_out=offset) == INVALID) == bool(out & first), offset


def test_steps_that_reach_past_all_memory(lib):
    s = {"q": (1 << 60, 64), "q_out": (1 << 61, 1 << 62), "k": (1 << 62, 64), "k_out": (64, 1 << 60)}
    assert passes(prompt(lib, layout(3, 2, 1 << 30, 64, s, 2), pos=1 << 50))       # (4 GB of positions)
