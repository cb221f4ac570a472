"""include/toploc_model.h without a GPU: every declared symbol is exported and bound, structs have the header's
sizes, and wrong arguments are refused before any CUDA call.  No kernel is launched here."""
import ctypes
import os
import re

import pytest
import torch

import paper_2501_16007_b200 as tl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = ctypes.c_void_p(1 << 20)          # an aligned address, never dereferenced here
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2501_16007_b200.csrc import build
    build.build()
    from paper_2501_16007_b200 import model_ops
    return model_ops._library()


def at(offset):
    return ctypes.c_void_p((1 << 20) + offset)


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "toploc_model.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(toploc_[a-z_]+)\s*\(", text)))
    assert "toploc_plan_pages" in names and len(names) >= 7
    for name in names:
        assert hasattr(lib, name), name
        assert hasattr(tl, name), "binding lacks %s" % name


def test_struct_sizes():
    assert ctypes.sizeof(tl.ToplocKvLayout) == 72
    assert ctypes.sizeof(tl.ToplocAttentionLayout) == 72
    assert ctypes.sizeof(tl.ToplocNormLayout) == 56


def test_status_strings(lib):
    texts = [tl.toploc_sequence_status_string(s) for s in range(7)]
    assert texts[0] == "ok" and len(set(texts)) == 7
    assert "unknown" in tl.toploc_sequence_status_string(77)


def plan(lib, **kw):
    a = dict(cached=OK, new=OK, n=4, free=OK, num_free=8, first=at(64), page=16, table=OK, width=4, stride=4, offs=OK,
             kv=OK, slots=OK, pos=OK, tokens=10, nxt=at(128), status=OK)
    a.update(kw)
    return lib.toploc_plan_pages(*a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(cached=None), INVALID), (dict(new=None), INVALID), (dict(first=None), INVALID), (dict(nxt=None), INVALID),
    (dict(nxt=at(64)), INVALID), (dict(slots=None), INVALID), (dict(slots=at(4)), INVALID), (dict(pos=at(2)), INVALID),
    (dict(table=None), INVALID), (dict(table=at(1)), INVALID), (dict(page=0), INVALID), (dict(n=-1), INVALID),
    (dict(stride=3), INVALID), (dict(tokens=-1), INVALID), (dict(num_free=-1), INVALID), (dict(status=None), INVALID),
    (dict(n=(1 << 24) + 1), UNSUPPORTED), (dict(tokens=1 << 31), UNSUPPORTED)])
def test_plan_refusals(lib, bad, code):
    assert plan(lib, **bad) == code


def kv_layout(**kw):
    base = dict(page_size=16, num_pages=8, max_pages=4, reserved=0, table_stride=4, k_page_stride=16 * 256,
                k_token_stride=256, k_head_stride=128, v_page_stride=16 * 256, v_token_stride=256, v_head_stride=128)
    base.update(kw)
    return tl.ToplocKvLayout(**base)


def write(lib, kv=None, **kw):
    a = dict(k=OK, v=OK, kt=256, kh=128, vt=256, vh=128, slots=OK, tokens=3, dtype=0, heads=2, dim=128, kc=OK, vc=OK)
    a.update(kw)
    return lib.toploc_cache_write(*a.values(), ctypes.byref(kv or kv_layout()), None)


@pytest.mark.parametrize("bad,code", [
    (dict(k=None), INVALID), (dict(vc=None), INVALID), (dict(slots=at(4)), INVALID), (dict(k=at(1)), INVALID),
    (dict(dtype=1, v=at(2)), INVALID), (dict(tokens=-1), INVALID), (dict(heads=0), INVALID), (dict(dim=0), INVALID),
    (dict(kt=-1), INVALID), (dict(dtype=5), UNSUPPORTED), (dict(kv=kv_layout(page_size=0)), INVALID)])
def test_write_refusals(lib, bad, code):
    assert write(lib, **bad) == code
    assert write(lib, tokens=0) == 0


def attention_layout(**kw):
    base = dict(dtype=0, head_dim=128, q_heads=8, kv_heads=2, num_seqs=3, max_new_tokens=4, total_tokens=12, scale=0.1,
                reserved=0, q_token_stride=1024, q_head_stride=128, out_token_stride=1024, out_head_stride=128)
    base.update(kw)
    return tl.ToplocAttentionLayout(**base)


def paged(lib, lay=None, kv=None, **kw):
    a = dict(q=OK, k=OK, v=OK, lay=ctypes.byref(lay or attention_layout()), kv=ctypes.byref(kv or kv_layout()),
             table=OK, offs=OK, lens=OK, out=OK, lse=None, status=None, ws=None, bytes=0)
    a.update(kw)
    return lib.toploc_attention_paged(*a.values(), None)


@pytest.mark.parametrize("lay,code", [
    (dict(head_dim=0), INVALID), (dict(kv_heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(num_seqs=-1), INVALID), (dict(max_new_tokens=-1), INVALID), (dict(q_token_stride=-8), INVALID),
    (dict(dtype=3), UNSUPPORTED), (dict(head_dim=12), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(q_heads=129 * 2), UNSUPPORTED), (dict(total_tokens=1 << 31), UNSUPPORTED)])
def test_attention_layout_refusals(lib, lay, code):
    bad = attention_layout(**lay)
    assert paged(lib, bad) == code
    flat = kv_layout(page_size=0)
    assert lib.toploc_attention_prompt(OK, OK, OK, ctypes.byref(bad), ctypes.byref(flat), OK, OK, None, None,
                                       None, 0, None) == code
    assert lib.toploc_attention_workspace_bytes(ctypes.byref(bad), ctypes.byref(kv_layout())) == 0


def test_attention_argument_refusals(lib):
    for name in ("q", "k", "v", "table", "offs", "lens", "out"):
        assert paged(lib, **{name: None}) == INVALID, name
    assert paged(lib, q=at(1)) == INVALID and paged(lib, offs=at(2)) == INVALID and paged(lib, lse=at(2)) == INVALID
    assert paged(lib, kv=kv_layout(page_size=0)) == INVALID
    assert paged(lib, kv=kv_layout(table_stride=2)) == INVALID
    assert paged(lib, kv=kv_layout(max_pages=1 << 28)) in (INVALID, UNSUPPORTED)
    assert paged(lib, lay=None, kv=None, ws=None) != 0 or not torch.cuda.is_available()
    assert lib.toploc_attention_paged(OK, OK, OK, None, None, OK, OK, OK, OK, None, None, None, 0, None) == INVALID
    for empty in (dict(num_seqs=0), dict(max_new_tokens=0), dict(total_tokens=0)):
        assert paged(lib, attention_layout(**empty)) == 0                       # nothing to do, nothing touched
    flat, lay = kv_layout(page_size=0), attention_layout()
    for i in (0, 1, 2, 5, 6):
        args = [OK, OK, OK, ctypes.byref(lay), ctypes.byref(flat), OK, OK, None, None, None, 0, None]
        args[i] = None
        assert lib.toploc_attention_prompt(*args) == INVALID, i
    assert lib.toploc_attention_prompt(OK, OK, OK, ctypes.byref(lay), ctypes.byref(kv_layout()), OK, OK, None, None,
                                       None, 0, None) == INVALID


def test_workspace(lib):
    def need(lay, kv):
        return lib.toploc_attention_workspace_bytes(ctypes.byref(lay), ctypes.byref(kv))
    long, one = kv_layout(max_pages=8192, table_stride=8192), dict(num_seqs=1, total_tokens=1, max_new_tokens=1)
    assert need(attention_layout(**one), long) >= 148 * 2 * 256 * 129 * 4       # parts of two row tiles a block
    assert need(attention_layout(dtype=1, **one), long) >= 2 * 8 * 129 * 4      # fp32: the keys in parts
    assert need(attention_layout(dtype=1, **one), kv_layout()) == 0
    assert need(attention_layout(dtype=1, num_seqs=4096, total_tokens=4096, max_new_tokens=1), long) == 0
    assert need(attention_layout(num_seqs=0), long) == 0


def norm(lib, lay=None, eps=1e-5, **kw):
    a = dict(x=OK, r=OK, w=OK, eps=eps, lay=ctypes.byref(lay or norm_layout()), ro=OK, y=OK, s=None)
    a.update(kw)
    return lib.toploc_rmsnorm_residual(*a.values(), None)


def norm_layout(**kw):
    base = dict(dtype=0, out_kind=0, group=0, hidden=64, rows=2, x_stride=64, residual_stride=64,
                residual_out_stride=64, y_stride=64)
    base.update(kw)
    return tl.ToplocNormLayout(**base)


def test_norm_refusals(lib):
    for name in ("x", "w", "y"):
        assert norm(lib, **{name: None}) == INVALID, name
    assert lib.toploc_rmsnorm_residual(OK, OK, OK, 1e-5, None, OK, OK, None, None) == INVALID
    assert norm(lib, norm_layout(out_kind=1)) == INVALID                        # e4m3 without scales
    assert norm(lib, norm_layout(out_kind=1), s=at(2)) == INVALID
    assert norm(lib, norm_layout(x_stride=63)) == INVALID and norm(lib, norm_layout(residual_stride=1)) == INVALID
    assert norm(lib, norm_layout(group=-1)) == INVALID and norm(lib, norm_layout(hidden=0)) == INVALID
    assert norm(lib, eps=-1.0) == INVALID and norm(lib, eps=float("nan")) == INVALID
    assert norm(lib, x=at(1)) == INVALID and norm(lib, norm_layout(dtype=1), ro=at(2)) == INVALID
    assert norm(lib, norm_layout(dtype=9)) == UNSUPPORTED and norm(lib, norm_layout(out_kind=7)) == UNSUPPORTED
    assert norm(lib, norm_layout(hidden=49160, x_stride=49160, residual_stride=49160, residual_out_stride=49160,
                                 y_stride=49160)) == UNSUPPORTED
    assert norm(lib, norm_layout(rows=0)) == 0


def test_wrappers_refuse_host_tensors_and_wrong_shapes():
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_rmsnorm_residual(x, x, x[0], 1e-5)
    with pytest.raises(tl.ToplocError, match="bfloat16 or float32"):
        tl.toploc_rmsnorm_residual(x.half(), None, x[0], 1e-5)
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_attention_prompt(q, q, q, torch.zeros(2, dtype=torch.int32), 4)
    cache = torch.zeros((2, 16, 2, 64), dtype=torch.bfloat16)
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_attention_paged(q, cache, cache, table, torch.zeros(2, dtype=torch.int32), lens, 4)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_cache_write(q, q, torch.zeros(4, dtype=torch.int64), cache, cache)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(tl.ToplocError, match="CUDA"):
        tl.toploc_plan_pages(i, i, i, i, table, 16, i, i, i.long(), i, i, i.byte())


def test_wrappers_refuse_numbers_that_do_not_fit():
    from paper_2501_16007_b200 import model_ops
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(tl.ToplocError, match="out of range"):
        model_ops._attention_layout(q, 2, 1, 1 << 40, None, q, None)
    lay = tl.ToplocAttentionLayout.from_buffer_copy(model_ops._attention_layout(q, 2, 3, 4, 0.25, q, None))
    assert (lay.head_dim, lay.q_heads, lay.kv_heads, lay.num_seqs, lay.max_new_tokens, lay.total_tokens, lay.scale,
            lay.q_token_stride, lay.out_head_stride) == (64, 2, 2, 3, 4, 4, 0.25, 128, 64)


def test_write_refuses_tokens_beyond_32_bits(lib):
    assert write(lib, heads=1 << 20, dim=1 << 11) == UNSUPPORTED        # 2^31 elements: places in a token would wrap
    assert write(lib, heads=(1 << 31) - 1, dim=(1 << 31) - 1) == UNSUPPORTED


def test_workspace_where_nothing_can_be_cut(lib):
    """Keys of at most three tiles stay with one block: room for its records, not for parts."""
    flat = kv_layout(page_size=0)
    for lay, kv, cut in [(dict(), kv_layout(max_pages=24, table_stride=24), False),
                         (dict(), kv_layout(max_pages=25, table_stride=25), True),
                         (dict(max_new_tokens=384, total_tokens=1000), flat, False),
                         (dict(max_new_tokens=385, total_tokens=1000), flat, True)]:
        need = lib.toploc_attention_workspace_bytes(ctypes.byref(attention_layout(**lay)), ctypes.byref(kv))
        assert need >= 148 * 2 * 256 * 129 * 4 if cut else 0 < need < 1 << 15, (lay, need)


def test_wait_limit_refusals(lib):
    assert paged(lib, attention_layout(wait_tries=-1)) == INVALID
    assert paged(lib, attention_layout(wait_tries=5, num_seqs=0)) == 0


def test_plan_refuses_outputs_in_inputs(lib):
    """Blocks read the lengths and the free list again while others write."""
    def call(**kw):                        # every array a megabyte from the next; 1000 sequences, tokens and pages
        names = ("cached", "new", "free", "first", "table", "offs", "kv", "slots", "pos", "nxt", "status")
        a = {name: at((2 + i) << 20) for i, name in enumerate(names)}
        a.update(kw)
        order = dict(cached=a["cached"], new=a["new"], n=1000, free=a["free"], num_free=1000, first=a["first"], page=16,
                     table=a["table"], width=4, stride=a.get("stride", 8), offs=a["offs"], kv=a["kv"], slots=a["slots"],
                     pos=a["pos"], tokens=1000, nxt=a["nxt"], status=a["status"])
        return lib.toploc_plan_pages(*order.values(), None)

    if not torch.cuda.is_available():                                   # (else they would run)
        assert call() not in (0, INVALID, UNSUPPORTED)                  # as far as the device
        for beside in (-1000, 1000):
            assert call(kv=at((2 << 20) + 4 * beside)) not in (0, INVALID)
        assert call(table=at(64 << 20), stride=1 << 62) not in (0, INVALID)
        # a vector between the rows of a table (of 4 entries, 4096 apart) shares nothing with it
        assert call(table=at(64 << 20), stride=4096, cached=at((64 << 20) + 64)) not in (0, INVALID)
    for name in ("cached", "new", "free"):
        where = (2 + ("cached", "new", "free").index(name)) << 20
        for out in ("offs", "kv", "slots", "pos", "nxt", "status", "table"):
            assert call(**{out: at(where)}) == INVALID, (name, out)
            assert call(**{out: at(where + 4 * 999 // 8 * 8)}) == INVALID, (name, out)
        assert call(kv=at(where - 4 * 999)) == INVALID and call(slots=at(where - 8 * 999)) == INVALID
        assert call(table=at(where - (8 * 999 + 3) * 4)) == INVALID
    first = 5 << 20
    for out in ("offs", "kv", "nxt", "status"):
        assert call(**{out: at(first)}) == INVALID
