"""Calls from several threads: the limits of a kernel are not one call's (the C calls run beside one another)."""
import threading

import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
CALLS = 3000


def together(*bodies):
    """Runs every body CALLS times on a thread and stream of its own; returns what was raised."""
    raised = []

    def run(body):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(CALLS):
                    body()
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            raised.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(b,)) for b in bodies]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return raised


def test_attention_of_two_head_sizes():
    offsets = torch.tensor([0, 5], dtype=torch.int32, device=DEV)
    bodies, outs, wants = [], [], []
    for dim in (96, 128, 104):
        q = torch.randn((5, 2, dim), device=DEV)
        out = torch.empty_like(q)
        wants.append(tl.toploc_attention_prompt(q, q, q, offsets, 5)[0])
        outs.append(out)
        bodies.append(lambda q=q, out=out: tl.toploc_attention_prompt(q, q, q, offsets, 5, out=out))
    assert not together(*bodies)
    assert all(torch.equal(a, b) for a, b in zip(outs, wants))


def test_norm_of_two_hidden_sizes():
    bodies, outs, wants = [], [], []
    for hidden in (12288, 49152, 24576):
        x, w = torch.randn((2, hidden), device=DEV), torch.ones(hidden, device=DEV)
        y = torch.empty((2, hidden), dtype=torch.float8_e4m3fn, device=DEV)
        scales = torch.empty((2, hidden // 48), device=DEV)
        wants.append(tl.toploc_rmsnorm_residual(x, None, w, 1e-5, group=48, quantize=True)[0])
        outs.append(y)
        bodies.append(lambda x=x, w=w, y=y, s=scales: tl.toploc_rmsnorm_residual(x, None, w, 1e-5, y=y, scales=s, group=48))
    assert not together(*bodies)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs, wants))


def test_final_norm_of_two_hidden_sizes():
    bodies, outs, wants = [], [], []
    for hidden in (20480, 81920, 40960):
        x, w = torch.randn((2, hidden), device=DEV).to(torch.bfloat16), torch.ones(hidden, device=DEV, dtype=torch.bfloat16)
        lay, _ = tl.make_layout(x, 1, 16, 2, 1)
        y = torch.empty_like(x)
        wants.append(tl.toploc_rmsnorm_append(x, w, 1e-5, lay, 0, torch.empty_like(x)))
        outs.append(y)
        bodies.append(lambda x=x, w=w, y=y, lay=lay: tl.toploc_rmsnorm_append(x, w, 1e-5, lay, 0, y))
    assert not together(*bodies)
    assert all(torch.equal(a, b) for a, b in zip(outs, wants))
