"""Norm with rotation, log probabilities and pools of pages without a GPU: structs have the header's sizes, wrong arguments
are refused before any CUDA call.  No kernel is launched here."""
import ctypes

import pytest
import torch

import paper_2501_16007_b200 as tl

INVALID, UNSUPPORTED = -1, -2
BASE = 1 << 24


def at(megabyte, offset=0):
    return ctypes.c_void_p(BASE + (megabyte << 20) + offset)


@pytest.fixture(scope="module")
def lib():
    from paper_2501_16007_b200.csrc import build
    build.build()
    from paper_2501_16007_b200 import model_ops
    return model_ops._library()


def passes(call, *args, **kw):
    """As far as the device: not refused for its arguments.  (On a machine with a GPU it would run: not called.)"""
    return torch.cuda.is_available() or call(*args, **kw) not in (0, INVALID, UNSUPPORTED)


def test_struct_sizes():
    assert ctypes.sizeof(tl.ToplocPoolLayout) == 48
    assert ctypes.sizeof(tl.ToplocRotaryLayout) == 120
    assert ctypes.sizeof(tl.ToplocLogprobLayout) == 32


def test_status_strings(lib):
    texts = [tl.toploc_sequence_status_string(s) for s in range(10)]
    assert len(set(texts)) == 10 and not any("unknown" in t for t in texts)


# ---- norm and rotation -----------------------------------------------------------------------------

def rotary_layout(**kw):
    base = dict(dtype=0, head_dim=128, q_heads=8, kv_heads=2, rotary_dim=128, pairing=0, num_tokens=3, eps=1e-6, reserved=0,
                q_token_stride=1024, q_head_stride=128, k_token_stride=256, k_head_stride=128, v_token_stride=256,
                v_head_stride=128, q_out_token_stride=1024, q_out_head_stride=128, k_out_token_stride=256,
                k_out_head_stride=128)
    base.update(kw)
    return tl.ToplocRotaryLayout(**base)


def kv_layout(**kw):
    base = dict(page_size=16, num_pages=8, max_pages=0, reserved=0, table_stride=0, k_page_stride=16 * 256,
                k_token_stride=256, k_head_stride=128, v_page_stride=16 * 256, v_token_stride=256, v_head_stride=128)
    base.update(kw)
    return tl.ToplocKvLayout(**base)


def prompt(lib, lay=None, **kw):
    a = dict(q=at(0), k=at(1), pos=at(2), freq=at(3), qw=at(4), kw=at(5), lay=ctypes.byref(lay or rotary_layout()), qo=at(6),
             ko=at(7))
    a.update(kw)
    return lib.toploc_norm_rotary_prompt(*a.values(), None)


def paged(lib, lay=None, kv=None, **kw):
    a = dict(q=at(0), k=at(1), v=at(8), pos=at(2), slots=at(9), freq=at(3), qw=at(4), kw=at(5),
             lay=ctypes.byref(lay or rotary_layout()), qo=at(6), kc=at(10), vc=at(11), kv=ctypes.byref(kv or kv_layout()))
    a.update(kw)
    return lib.toploc_norm_rotary_paged(*a.values(), None)


@pytest.mark.parametrize("lay,code", [
    (dict(head_dim=0), INVALID), (dict(q_heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(rotary_dim=-2), INVALID),
    (dict(rotary_dim=127), INVALID), (dict(rotary_dim=130), INVALID), (dict(pairing=2), INVALID),
    (dict(pairing=-1), INVALID), (dict(num_tokens=-1), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(q_token_stride=-8), INVALID), (dict(k_head_stride=-8), INVALID),
    (dict(q_out_head_stride=-8), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(head_dim=257, rotary_dim=2), UNSUPPORTED),
    (dict(num_tokens=1 << 31), UNSUPPORTED), (dict(q_heads=16385), UNSUPPORTED)])
def test_rotary_layout_refusals(lib, lay, code):
    assert prompt(lib, rotary_layout(**lay)) == code
    assert paged(lib, rotary_layout(**lay)) == code


def test_rotary_argument_refusals(lib):
    assert passes(prompt, lib) and passes(paged, lib)
    for name in ("q", "k", "pos", "freq", "qo"):
        assert prompt(lib, **{name: None}) == INVALID, name
        assert paged(lib, **{name: None}) == INVALID, name
    for name in ("v", "slots", "kc", "vc"):
        assert paged(lib, **{name: None}) == INVALID, name
    assert prompt(lib, ko=None) == INVALID and passes(prompt, lib, qw=None, kw=None)
    assert prompt(lib, q=at(0, 1)) == INVALID and prompt(lib, pos=at(2, 2)) == INVALID and prompt(lib, kw=at(5, 1)) == INVALID
    assert prompt(lib, freq=at(3, 2)) == INVALID and paged(lib, slots=at(9, 4)) == INVALID
    assert paged(lib, kv=kv_layout(page_size=0)) == INVALID and paged(lib, kv=kv_layout(num_pages=-1)) == INVALID
    assert paged(lib, kv=kv_layout(v_page_stride=-1)) == INVALID
    assert prompt(lib, rotary_layout(num_tokens=0), q=None) == 0
    assert passes(prompt, lib, qo=at(0), ko=at(1))                                     # in place
    assert prompt(lib, rotary_layout(q_out_token_stride=2048), qo=at(0)) == INVALID    # but every head at its own place
    assert prompt(lib, rotary_layout(k_out_head_stride=256), ko=at(1)) == INVALID
    assert paged(lib, rotary_layout(q_out_head_stride=256), qo=at(0)) == INVALID
    assert passes(prompt, lib, rotary_layout(rotary_dim=0), pos=None, freq=None)       # nothing turns
    assert lib.toploc_norm_rotary_prompt(at(0), at(1), at(2), at(3), None, None, None, at(6), at(7), None) == INVALID


def test_rotary_wrapper_refusals():
    q, k = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros((4, 1, 64), dtype=torch.bfloat16)
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(32)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_norm_rotary_prompt(q, k, i, f)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_norm_rotary_paged(q, k, k, i, i.long(), f, torch.zeros((2, 16, 1, 64)), torch.zeros((2, 16, 1, 64)))
    from paper_2501_16007_b200 import model_ops

    def layout(**kw):
        a = dict(q=q, k=k, v=None, positions=i, inv_freq=f, q_weight=None, k_weight=None, eps=0.0, pairing="halves",
                 q_out=q, k_out=k)
        a.update(kw)
        return model_ops._rotary_layout(**a)

    lay = tl.ToplocRotaryLayout.from_buffer_copy(layout(v=k, pairing="neighbours"))
    assert (lay.head_dim, lay.q_heads, lay.kv_heads, lay.rotary_dim, lay.pairing, lay.num_tokens, lay.q_token_stride,
            lay.v_head_stride, lay.k_out_token_stride) == (64, 2, 1, 64, 1, 4, 128, 64, 64)
    for bad in (dict(k=k.float()), dict(k=k[:3]), dict(positions=i[:3]), dict(positions=i.long()), dict(inv_freq=f.double()),
                dict(inv_freq=torch.zeros(33)), dict(pairing="other"), dict(q_weight=torch.zeros(64)),
                dict(q_weight=torch.zeros(63, dtype=torch.bfloat16)), dict(q_out=q[:, :1]), dict(k_out=k.float()),
                dict(v=k[:, :, :32]), dict(q=q.half(), q_out=q.half()), dict(q=q.transpose(1, 2))):
        with pytest.raises(tl.ToplocError):
            layout(**bad)


# ---- log probabilities -----------------------------------------------------------------------------

def logprobs(lib, lay=None, **kw):
    a = dict(x=at(0), lay=ctypes.byref(lay or logprob_layout()), tokens=at(1), lp=at(2), h=at(3), ids=at(4), top=at(5))
    a.update(kw)
    return lib.toploc_token_logprobs(*a.values(), None)


def logprob_layout(**kw):
    base = dict(dtype=0, vocab=1000, top=5, reserved=0, rows=4, row_stride=1000)
    base.update(kw)
    return tl.ToplocLogprobLayout(**base)


@pytest.mark.parametrize("lay,code", [
    (dict(vocab=0), INVALID), (dict(vocab=-1), INVALID), (dict(top=-1), INVALID), (dict(rows=-1), INVALID),
    (dict(row_stride=999), INVALID), (dict(dtype=4), UNSUPPORTED), (dict(top=33), UNSUPPORTED),
    (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED)])
def test_logprob_layout_refusals(lib, lay, code):
    assert logprobs(lib, logprob_layout(**lay)) == code


def test_logprob_argument_refusals(lib):
    assert passes(logprobs, lib) and passes(logprobs, lib, tokens=None, lp=None, h=None)
    assert lib.toploc_token_logprobs(at(0), None, None, None, None, None, None, None) == INVALID
    for bad in (dict(x=None), dict(tokens=None), dict(lp=None), dict(ids=None), dict(top=None), dict(x=at(0, 1)),
                dict(tokens=at(1, 4)), dict(lp=at(2, 2)), dict(h=at(3, 2)), dict(ids=at(4, 4)), dict(top=at(5, 2))):
        assert logprobs(lib, **bad) == INVALID, bad
    assert logprobs(lib, logprob_layout(dtype=1), x=at(0, 2)) == INVALID
    assert passes(logprobs, lib, logprob_layout(top=0), ids=None, top=None)
    assert logprobs(lib, logprob_layout(rows=0), x=None) == 0


def test_logprob_wrapper_refusals():
    x, t = torch.zeros((3, 50)), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_token_logprobs(x, t)
    for bad in (dict(logits=x.half()), dict(logits=x[0]), dict(logits=x.t()), dict(top=-1), dict(logprobs=x[:, 0]),
                dict(top_ids=t[:, None]), dict(top=2, top_ids=t[:, None]), dict(top=2, top_logprobs=x[:, :2].double())):
        a = dict(logits=x)
        a.update(bad)
        with pytest.raises(tl.ToplocError):
            tl.toploc_token_logprobs(**a)


# ---- pools -----------------------------------------------------------------------------------------

FORK = ("parents", "lens", "n", "shares", "pages", "free", "num_free", "first", "page", "table", "width", "stride",
        "lens_out", "shares_out", "source", "target", "copies", "next", "status")
RELEASE = ("release", "lens", "n", "table", "width", "stride", "shares", "pages", "page", "free", "num_free", "first",
           "lens_out", "shares_out", "next", "status")
COMPACT = ("lens", "n", "table", "width", "stride", "shares", "pages", "page", "table_out", "stride_out", "shares_out",
           "free", "num_free", "source", "target", "copies", "next", "status")
NUMBERS = dict(n=1000, pages=1000, num_free=1000, page=16, width=4, stride=8, stride_out=8)
PLANNERS = [("toploc_fork_pages", FORK, ("parents", "lens", "shares", "free", "first")),
            ("toploc_release_pages", RELEASE, ("release", "lens", "table", "shares", "first")),
            ("toploc_compact_pages", COMPACT, ("lens", "table", "shares"))]


def planner(lib, name, order, **kw):
    """Every array a megabyte from the next."""
    a = {k: NUMBERS.get(k, at(i)) for i, k in enumerate(order)}
    a.update(kw)
    return getattr(lib, name)(*[a[k] for k in order], None)


@pytest.mark.parametrize("name,order,inputs", PLANNERS)
def test_planner_refusals(lib, name, order, inputs):
    assert passes(planner, lib, name, order)
    arrays = [k for k in order if k not in NUMBERS]
    for k in arrays:
        assert planner(lib, name, order, **{k: None}) == INVALID, k
        if k not in ("release", "status"):
            assert planner(lib, name, order, **{k: at(order.index(k), 2)}) == INVALID, k
    for bad in (dict(n=-1), dict(pages=-1), dict(num_free=-1), dict(page=0), dict(width=-1), dict(stride=3)):
        assert planner(lib, name, order, **bad) == INVALID, bad
    assert planner(lib, name, order, n=(1 << 24) + 1) == UNSUPPORTED
    if name != "toploc_compact_pages":
        assert planner(lib, name, order, pages=(1 << 30) + 1) == UNSUPPORTED
    else:
        assert planner(lib, name, order, stride_out=3) == INVALID and planner(lib, name, order, num_free=999) == INVALID


@pytest.mark.parametrize("name,order,inputs", PLANNERS)
def test_planners_refuse_outputs_in_other_arrays(lib, name, order, inputs):
    """Blocks read inputs again while others write; in_place is the compacted table's alone."""
    arrays = [k for k in order if k not in NUMBERS]
    for out in (k for k in arrays if k not in inputs):
        for other in arrays:
            if other == out or (out, other) == ("table_out", "table"):
                continue
            assert planner(lib, name, order, **{out: at(order.index(other))}) == INVALID, (out, other)
    if name == "toploc_compact_pages":
        table = order.index("table")
        assert passes(planner, lib, name, order, table_out=at(table))
        assert planner(lib, name, order, table_out=at(table), stride_out=9) == INVALID
        assert planner(lib, name, order, table_out=at(table, 4)) == INVALID
        assert passes(planner, lib, name, order, table_out=at(table, 16))      # between its rows
        assert planner(lib, name, order, table_out=at(table, 20)) == INVALID   # into the next one
        assert passes(planner, lib, name, order, table_out=at(table + 40), stride_out=1 << 50)


def test_planner_wrapper_refusals():
    i, b, t = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.uint8), torch.zeros((3, 2), dtype=torch.int32)
    one = i[:1]
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_fork_pages(i, i, i, i, one, t, 16, i, i, i, i, one, one, b)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_release_pages(b, i, t, i, 16, i, one, i, i, one, b)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_compact_pages(i, t, i, 16, t, i, i, i, i, one, one, b)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_copy_pages([torch.zeros((2, 16, 2, 64))], i, i, one)
    tl.toploc_copy_pages([], i, i, one)


def pool_layout(**kw):
    base = dict(dtype=0, num_pages=8, page_size=16, kv_heads=2, head_dim=64, num_caches=2, page_stride=2048, token_stride=128,
                head_stride=64)
    base.update(kw)
    return tl.ToplocPoolLayout(**base)


def copy(lib, lay=None, caches=(1, 2), **kw):
    pointers = (ctypes.c_void_p * len(caches))(*[None if c is None else BASE + c for c in caches])
    a = dict(caches=pointers, lay=ctypes.byref(lay or pool_layout()), source=at(3), target=at(4), count=at(5), most=10)
    a.update(kw)
    return lib.toploc_copy_pages(*a.values(), None)


def test_copy_refusals(lib):
    even = (0, 1 << 20)
    assert passes(copy, lib, caches=even)
    for bad in (dict(num_pages=-1), dict(page_size=0), dict(kv_heads=0), dict(head_dim=0), dict(num_caches=-1),
                dict(page_stride=-1), dict(token_stride=-1), dict(head_stride=-1)):
        assert copy(lib, pool_layout(**bad), even) == INVALID, bad
    assert copy(lib, pool_layout(dtype=7), even) == UNSUPPORTED
    assert copy(lib, pool_layout(kv_heads=1 << 20, head_dim=1 << 11), even) == UNSUPPORTED
    for bad in (dict(source=None), dict(target=None), dict(count=None), dict(most=-1), dict(source=at(3, 2)),
                dict(target=at(4, 1)), dict(count=at(5, 2))):
        assert copy(lib, caches=even, **bad) == INVALID, bad
    assert lib.toploc_copy_pages(None, ctypes.byref(pool_layout()), at(3), at(4), at(5), 10, None) == INVALID
    assert lib.toploc_copy_pages((ctypes.c_void_p * 2)(), None, at(3), at(4), at(5), 10, None) == INVALID
    assert copy(lib, caches=(0, None)) == INVALID and copy(lib, caches=(0, 1)) == INVALID
    assert copy(lib, pool_layout(dtype=1), (0, 2)) == INVALID
    assert copy(lib, pool_layout(num_caches=0), ()) == 0 and copy(lib, caches=even, most=0) == 0
