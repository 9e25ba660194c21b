"""The example that runs the training operators together."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "finetune.py")
    spec = importlib.util.spec_from_file_location("finetune", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_loss_falls(example, dtype):
    losses = example.finetune(dtype=dtype)
    assert losses[0] > 5.0                      # log 1000 = 6.9: nothing is known yet
    assert losses[-1] < 0.5 * losses[0]


def test_types_start_alike(example):
    # logits are of order one and pass five roundings to bf16 of 2^-9 each
    a, b = (example.finetune(steps=1, dtype=t)[0] for t in (torch.float32, torch.bfloat16))
    assert abs(a - b) < 0.05


def test_repeats_exactly(example):
    assert example.finetune(steps=5) == example.finetune(steps=5)
