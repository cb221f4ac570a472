"""Memory that a call allocates belongs to the stream it was given (no GPU: the allocator's streams are stood in for).

A block allocated on torch's current stream and dropped on return would go to the next allocation of the current stream,
while the kernels on the given stream still write to it."""
import contextlib

import pytest
import torch

import paper_2501_16007_b200 as tl
from paper_2501_16007_b200 import binding, model_ops


class Named:
    """Something that names a CUDA stream and is none of torch's."""

    def __init__(self, handle):
        self.cuda_stream = handle


CURRENT, SIDE = Named(0), Named(77)


@pytest.fixture
def allocations(monkeypatch):
    """[(shape, stream that was current at the allocation, streams recorded later)]"""
    made, now, empty = [], [CURRENT], torch.empty

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def recorded_empty(*shape, **kw):
        t = empty(*shape, **dict(kw, device="cpu"))
        made.append((t, now[-1], []))
        return t

    def record(t, stream):
        for other, _, streams in made:
            if other is t:
                streams.append(stream)

    monkeypatch.setattr(torch, "empty", recorded_empty)
    monkeypatch.setattr(torch, "empty_like", lambda t, **kw: recorded_empty(t.shape, dtype=t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: {77: SIDE}[handle])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", record)
    return made


def check(made, shapes, stream):
    """All allocations were made on `stream`; what the caller gets is also kept for the current one."""
    assert sorted(tuple(t.shape) for t, _, _ in made) == sorted(shapes)
    for t, where, recorded in made:
        assert where == stream, "%s allocated on stream %d" % (tuple(t.shape), where.cuda_stream)
        if stream != CURRENT:
            assert recorded == ([] if t.shape == (640,) else [CURRENT]), tuple(t.shape)   # 640: the workspace


class Library:
    def __getattr__(self, name):
        return lambda *args: 640 if name.endswith("bytes") else 0


@pytest.mark.parametrize("given,expected", [(None, CURRENT), (CURRENT, CURRENT), (SIDE, SIDE)])
def test_model_operators(monkeypatch, allocations, given, expected):
    monkeypatch.setattr(model_ops, "_library", Library)
    monkeypatch.setattr(model_ops, "_device", lambda name, *tensors: tensors[0].device)
    monkeypatch.setattr(model_ops, "_call", lambda *args: None)
    q, kv = torch.zeros((4, 8, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    cache, i32 = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16), torch.int32
    table, offsets, lens = torch.zeros((1, 3), dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32)
    del allocations[:]
    tl.toploc_attention_paged(q, cache, cache, table, offsets, lens, 4, want_lse=True, stream=given)
    check(allocations, [(4, 8, 64), (4, 8), (640,)], expected)
    del allocations[:]
    tl.toploc_attention_prompt(q, kv, kv, offsets, 4, want_lse=True, stream=given)
    check(allocations, [(4, 8, 64), (4, 8), (640,)], expected)
    x, w = torch.zeros((4, 512), dtype=torch.bfloat16), torch.zeros(512, dtype=torch.bfloat16)
    del allocations[:]
    tl.toploc_rmsnorm_residual(x, x, w, 1e-5, quantize=True, group=128, stream=given)
    check(allocations, [(4, 512), (4, 512), (4, 4)], expected)


@pytest.mark.parametrize("given,expected", [(None, CURRENT), (CURRENT, CURRENT), (SIDE, SIDE)])
def test_proof_path(monkeypatch, allocations, given, expected):
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "toploc_num_chunks", lambda lay: 2)
    monkeypatch.setattr(binding, "toploc_stream_workspace_bytes", lambda lay: 640)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "device", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    act = torch.zeros((64, 256), dtype=torch.bfloat16)
    lay, _ = tl.make_layout(act, 32, 16, 2, 32)
    proofs, thr = torch.zeros((2, 640), dtype=torch.uint8), tl.ToplocThresholds()
    per_chunk = torch.zeros((2, 24), dtype=torch.uint8)
    state = torch.zeros(64, dtype=torch.uint8)
    commits = torch.zeros((2, 96), dtype=torch.uint8)
    for call, shapes in [
            (lambda: tl.toploc_build_proofs(act, lay, want_indices=True, stream=given), [(2, 640), (2,), (2, 16), (640,)]),
            (lambda: tl.toploc_verify_proofs(act, lay, proofs, thr, stream=given), [(2, 40), (640,)]),
            (lambda: tl.toploc_verify_proofs_per_chunk_thresholds(act, lay, proofs, per_chunk, stream=given),
             [(2, 40), (640,)]),
            (lambda: tl.toploc_select_topk(act, lay, want_ranked=True, stream=given),
             [(2, 16), (2, 16), (2,), (2, 16), (640,)]),
            (lambda: tl.toploc_stream_finish(state, lay, want_indices=True, stream=given),
             [(2, 640), (2,), (2, 16), (640,)]),
            (lambda: tl.toploc_commit_direct(act, lay, stream=given), [(2, 96), (2,)]),
            (lambda: tl.toploc_verify_direct(act, lay, commits, thr, stream=given), [(2, 40), (2, 9)]),
            (lambda: tl.toploc_verify_direct_per_chunk_thresholds(act, lay, commits, per_chunk, stream=given),
             [(2, 40), (2, 9)])]:
        del allocations[:]
        call()
        check(allocations, shapes, expected)
