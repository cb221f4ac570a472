"""Attention where a sequence is longer than the call was told, or rows belong to no sequence: those rows stay as they are,
whatever lies in the workspace, with every kernel."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype,dim", [(torch.float32, 64), (torch.bfloat16, 96), (torch.bfloat16, 128)])
@pytest.mark.parametrize("offsets,most,kept", [([0, 3, 10, 12], 3, [(6, 10)]),    # the second sequence is clipped to 3 rows
                                               ([4, 6, 7, 10], 3, [(0, 4)])])     # the first four rows are nobody's
def test_rows_outside_the_promised_ones_stay(dtype, dim, offsets, most, kept):
    g = torch.Generator(device=DEV)
    g.manual_seed(dim + most)
    page, pages, rows = 64, 40, offsets[-1] + 2
    kv = [2000, 2500, 1000]
    caches = [torch.randn((pages, page, 2, dim), generator=g, device=DEV).to(dtype) for _ in range(2)]
    table = torch.randint(0, pages, (3, pages), generator=g, device=DEV, dtype=torch.int32)   # wide: keys are split
    q = torch.randn((rows, 8, dim), generator=g, device=DEV).to(dtype)
    out, lse = torch.full_like(q, 7.0), torch.full((rows, 8), 7.0, device=DEV)
    status = torch.zeros(3, dtype=torch.uint8, device=DEV)
    need = tl.toploc_attention_workspace_bytes(q, *caches, table, most)
    assert need > 0
    work = torch.full((need,), 0x3C, dtype=torch.uint8, device=DEV)              # what an earlier call may have left
    i32 = dict(dtype=torch.int32, device=DEV)
    tl.toploc_attention_paged(q, *caches, table, torch.tensor(offsets, **i32), torch.tensor(kv, **i32), most, out=out,
                              lse=lse, status=status, workspace=work)
    for a, b in kept + [(offsets[-1], rows)]:
        assert (out[a:b] == 7.0).all() and (lse[a:b] == 7.0).all()
    written = torch.ones(rows, dtype=torch.bool)
    for a, b in kept + [(offsets[-1], rows)]:
        written[a:b] = False
    assert (lse[written.to(DEV)] != 7.0).all() and not torch.isnan(out).any()
    lens = [b - a for a, b in zip(offsets, offsets[1:])]
    assert status.tolist() == [tl.TOPLOC_SEQ_BAD_LENGTH if n > most else 0 for n in lens]


@pytest.mark.parametrize("keys,new,heads,kv_heads,dim", [(384, 1, 8, 2, 128), (384, 40, 8, 2, 64), (384, 384, 4, 2, 128),
                                                         (300, 7, 4, 4, 64), (6000, 1, 8, 2, 64), (6000, 40, 8, 2, 128)])
def test_nothing_behind_the_workspace_is_written(keys, new, heads, kv_heads, dim):
    g = torch.Generator(device=DEV)
    g.manual_seed(keys + dim)
    page, n = 16, 9
    pages = -(-keys // page)
    caches = [torch.randn((pages, page, kv_heads, dim), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]
    table = torch.randint(0, pages, (n, pages), generator=g, device=DEV, dtype=torch.int32)
    q = torch.randn((n * new, heads, dim), generator=g, device=DEV).to(torch.bfloat16)
    i32 = dict(dtype=torch.int32, device=DEV)
    args = (q, *caches, table, torch.arange(0, n * new + 1, new, **i32), torch.full((n,), keys, **i32), new)
    want = tl.toploc_attention_paged(*args, want_lse=True)
    need = tl.toploc_attention_workspace_bytes(*args[:4], new)
    room = torch.full((need + (1 << 20),), 0x3C, dtype=torch.uint8, device=DEV)
    got = tl.toploc_attention_paged(*args, want_lse=True, workspace=room[:need])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (room[need:] == 0x3C).all()
