"""Calls on side streams that allocate their own workspaces and outputs: results are those of serial calls, bit for bit."""
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def problem(seed, keys, new, heads, kv_heads, dim, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    pages = -(-keys // 64)
    caches = [torch.randn((pages, 64, kv_heads, dim), generator=g, device=DEV).to(dtype) for _ in range(2)]
    q = torch.randn((new, heads, dim), generator=g, device=DEV).to(dtype)
    table = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).view(1, pages)
    i32 = torch.int32
    return q, *caches, table, torch.tensor([0, new], dtype=i32, device=DEV), torch.tensor([keys], dtype=i32, device=DEV), new


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_on_two_side_streams_without_workspaces(dtype):
    """Keys cut over blocks, so that both calls write parts; allocations on the current stream behind them."""
    first = problem(1, 20000, 17, 16, 2, 128, dtype)
    second = problem(2, 9000, 1, 8, 2, 64, dtype)
    want = [tl.toploc_attention_paged(*p, want_lse=True) for p in (first, second)]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        got = []
        for side, p in zip(sides, (first, second)):
            got.append(tl.toploc_attention_paged(*p, want_lse=True, stream=side))
            # a block of the workspace's size on the current stream, written at once
            need = tl.toploc_attention_workspace_bytes(p[0], p[1], p[2], p[3], p[6])
            torch.empty(need, dtype=torch.uint8, device=DEV).fill_(0xA5)
        torch.cuda.synchronize()
        for (out, lse), (out_want, lse_want) in zip(got, want):
            assert torch.equal(out, out_want) and torch.equal(lse, lse_want)


def test_norm_on_a_side_stream_behind_frees_of_the_current_one():
    """Outputs of the call do not take memory that the current stream still writes to."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn((4096, 4096), generator=g, device=DEV).to(torch.bfloat16)
    w = torch.ones(4096, dtype=torch.bfloat16, device=DEV)
    want = tl.toploc_rmsnorm_residual(x, None, w, 1e-5)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(20):
        busy = torch.empty_like(x)
        for _ in range(10):
            busy.fill_(7.0)
        del busy                                        # the current stream writes to it for a while yet
        got = tl.toploc_rmsnorm_residual(x, None, w, 1e-5, stream=side)[0]
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_a_stream_that_is_not_torchs():
    """An object with the handle of a CUDA stream, as other libraries have them."""
    class Named:
        cuda_stream = torch.cuda.Stream().cuda_stream

    x = torch.randn((64, 512), device=DEV)
    w = torch.ones(512, device=DEV)
    want = tl.toploc_rmsnorm_residual(x, None, w, 1e-5)[0]
    torch.cuda.synchronize()
    got = tl.toploc_rmsnorm_residual(x, None, w, 1e-5, stream=Named())[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
