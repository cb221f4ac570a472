"""A workspace has the bytes that the call is told: an expanded or strided tensor is refused (no GPU: calls are stood in for)."""
import contextlib

import pytest
import torch

import paper_2501_16007_b200 as tl
from paper_2501_16007_b200 import binding, model_ops


class Library:
    def __getattr__(self, name):
        return lambda *args: 640 if name.endswith("bytes") else 0


@pytest.mark.parametrize("workspace,fits", [(torch.zeros(640, dtype=torch.uint8), True),
                                            (torch.zeros(1, dtype=torch.uint8).expand(640), False),
                                            (torch.zeros((2, 1000), dtype=torch.uint8)[:, :320], False)])
def test_workspaces(monkeypatch, workspace, fits):
    monkeypatch.setattr(model_ops, "_library", Library)
    monkeypatch.setattr(model_ops, "_device", lambda name, *tensors: tensors[0].device)
    monkeypatch.setattr(model_ops, "_call", lambda *args: None)
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "toploc_num_chunks", lambda lay: 2)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "device", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    cache, lens = torch.zeros((2, 16, 2, 64), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    table, offsets = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    act = torch.zeros((64, 256), dtype=torch.bfloat16)
    lay, _ = tl.make_layout(act, 32, 16, 2, 32)
    proofs, state = torch.zeros((2, 640), dtype=torch.uint8), torch.zeros(64, dtype=torch.uint8)
    thresholds = tl.ToplocThresholds()
    for call in (lambda: tl.toploc_attention_paged(q, cache, cache, table, offsets, lens, 4, workspace=workspace),
                 lambda: tl.toploc_attention_prompt(q, q, q, offsets, 4, workspace=workspace),
                 lambda: tl.toploc_build_proofs(act, lay, workspace=workspace),
                 lambda: tl.toploc_verify_proofs(act, lay, proofs, thresholds, workspace=workspace),
                 lambda: tl.toploc_select_topk(act, lay, workspace=workspace),
                 lambda: tl.toploc_stream_finish(state, lay, workspace=workspace)):
        if fits:
            call()
        else:
            with pytest.raises(tl.ToplocError, match="contiguous"):
                call()
