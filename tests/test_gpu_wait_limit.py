"""Waits inside the tensor-core kernels that run out (a limit of one try, so that some always do): the call returns, copies
and products in flight have ended, tensor memory is free again, and the calls behind it are right."""
import ctypes

import pytest
import torch

import paper_2501_16007_b200 as tl
from paper_2501_16007_b200 import model_ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32


def ints(values):
    return torch.tensor(values, dtype=I32, device=DEV)


class Paged:
    """Sequences over scattered pages, each behind `idle` ones without new tokens (the warp that looks for the work passes
    them one by one, so the others wait for many tries), and the call through the C entry with a limit of its waits."""

    def __init__(self, kv, new, heads, kv_heads, dim, idle=30000, page=64):
        g = torch.Generator(device=DEV)
        g.manual_seed(len(kv) + dim)
        self.every, self.n = idle + 1, len(kv) * (idle + 1)
        width = max(-(-c // page) for c in kv)
        pages = width * len(kv)
        self.caches = [torch.randn((pages, page, kv_heads, dim), generator=g, device=DEV).to(torch.bfloat16)
                       for _ in range(2)]
        self.table = torch.zeros((self.n, width), dtype=I32, device=DEV)
        self.table[idle::self.every] = torch.randperm(pages, generator=g, device=DEV).to(I32).view(len(kv), width)
        lens, rows = torch.zeros(self.n, dtype=I32), torch.zeros(self.n, dtype=I32)
        lens[idle::self.every], rows[idle::self.every] = torch.tensor(kv, dtype=I32), torch.tensor(new, dtype=I32)
        self.offsets = torch.cat([torch.zeros(1, dtype=I32), rows.cumsum(0).to(I32)])
        self.q = torch.randn((sum(new), heads, dim), generator=g, device=DEV).to(torch.bfloat16)
        self.most = max(new)
        self.args = (self.q, *self.caches, self.table, self.offsets.to(DEV), lens.to(DEV), self.most)
        self.out = torch.empty_like(self.q)
        self.lse = torch.empty(self.q.shape[:2], device=DEV)
        self.status = torch.empty(self.n, dtype=torch.uint8, device=DEV)
        self.work = torch.empty(tl.toploc_attention_workspace_bytes(*self.args[:4], self.most), dtype=torch.uint8,
                                device=DEV)

    def call(self, wait_tries):
        self.out.fill_(7.0)
        self.lse.fill_(7.0)
        self.status.zero_()
        lay = tl.ToplocAttentionLayout.from_buffer_copy(model_ops._attention_layout(
            self.q, self.caches[0].shape[2], self.n, self.most, None, self.out, self.lse))
        lay.wait_tries = wait_tries
        kv = model_ops._cache_layout(*self.caches, self.table)
        q, k, v, table, offsets, lens, _ = self.args
        rc = model_ops._library().toploc_attention_paged(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(lay), kv, table.data_ptr(), offsets.data_ptr(),
            lens.data_ptr(), self.out.data_ptr(), self.lse.data_ptr(), self.status.data_ptr(), self.work.data_ptr(),
            self.work.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        torch.cuda.synchronize()


CASES = [([5000, 130, 2049, 64, 777], [32, 1, 64, 64, 10], 16, 2, 128),    # many rows
         ([3000, 1000], [100, 40], 8, 2, 64),
         ([20000], [17], 64, 8, 128),                                      # one sequence over all blocks
         ([5000, 130, 2049, 64, 777] * 4, [1] * 20, 8, 2, 128),            # few rows
         ([40000], [1], 8, 2, 64)]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_the_call_returns_and_the_next_one_is_right(case):
    p = Paged(*CASES[case])
    want = tl.toploc_attention_paged(*p.args, want_lse=True)
    torch.cuda.synchronize()
    for _ in range(5):
        p.call(1)
        assert (p.status == tl.TOPLOC_SEQ_WAIT_EXPIRED).any()
        p.call(0)
        assert not p.status.any()
        assert torch.equal(p.out, want[0]) and torch.equal(p.lse, want[1])


@pytest.mark.parametrize("case", range(len(CASES)))
def test_expired_waits_show_on_the_rows_and_sequences_they_spoil(case):
    p = Paged(*CASES[case])
    p.call(0)
    want_out, want_lse = p.out.clone(), p.lse.clone()
    assert not p.status.any() and not torch.isnan(want_lse).any()
    lens = p.offsets[1:] - p.offsets[:-1]
    sequence = torch.repeat_interleave(torch.arange(p.n), lens).to(DEV)       # of every row
    for _ in range(5):
        p.work.fill_(0x3C)                                # what an earlier call may have left there
        p.call(1)
        flagged = p.status == tl.TOPLOC_SEQ_WAIT_EXPIRED
        assert flagged.any() and ((p.status == 0) | flagged).all()
        assert (lens.to(DEV)[flagged] > 0).all(), "a sequence without rows is flagged"
        nan = torch.isnan(p.lse)
        assert torch.equal(torch.where(nan, want_lse, p.lse), want_lse), "a row neither right nor NaN"
        assert torch.equal(torch.where(nan[:, :, None], want_out, p.out), want_out)
        assert torch.isnan(p.out[nan]).all()
        assert flagged[sequence[nan.any(1)]].all(), "a spoilt row whose sequence is not flagged"
        assert nan.any()
