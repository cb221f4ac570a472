"""The example notices what its calls flag."""
import importlib.util
import os

import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "provider_and_validator.py")


def load():
    spec = importlib.util.spec_from_file_location("provider_and_validator", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_a_provider_without_pages_raises():
    example = load()
    prompts = [[1, 2, 3], [4] * 40]
    provider = example.Provider(example.Model(1, "cuda"), 2, 40, torch.device("cuda"))
    provider.free = provider.free[:4]                    # the prompts' pages and no more: both run out on the way
    with pytest.raises(tl.ToplocError, match="free list exhausted"):
        provider.generate(prompts)


def test_a_provider_whose_table_is_damaged_raises():
    example = load()
    prompts = [[1, 2, 3], [4] * 40]
    provider = example.Provider(example.Model(1, "cuda"), 2, 40, torch.device("cuda"))
    provider.step(torch.tensor([p for q in prompts for p in q], device="cuda"),
                  torch.zeros(2, dtype=torch.int32, device="cuda"),
                  torch.tensor([3, 40], dtype=torch.int32, device="cuda"), 40)
    example.check_status(provider.status)
    provider.table[1, 0] = 10 ** 6
    provider.step(torch.tensor([5, 6], device="cuda"), torch.tensor([3, 40], dtype=torch.int32, device="cuda"),
                  torch.ones(2, dtype=torch.int32, device="cuda"), 1)
    with pytest.raises(tl.ToplocError, match="sequence 1: block table entry outside the cache"):
        example.check_status(provider.status)
