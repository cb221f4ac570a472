"""The model-side operators together, as a provider and a validator use them: ragged prompts and 32 decode steps over a
paged cache with proofs on one side, one packed pass and the verdicts on the other."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "provider_and_validator.py")


def test_honest_proofs_pass_and_other_weights_fail():
    spec = importlib.util.spec_from_file_location("provider_and_validator", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    honest, other = example.main()
    assert honest["accept"].all() and not honest["status"].any()
    assert not other["accept"].any()
