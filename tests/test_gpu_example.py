"""The 8-bit training example end to end: it learns, the same seed gives the same losses, and single tokens served from
held weights are the batch's rows."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "train_fp8.py"
    spec = importlib.util.spec_from_file_location("train_fp8", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns_and_serves(example):
    losses, weights, x, target = example.train(steps=120)
    assert losses[-1] < 0.5 * losses[0]
    again = example.train(steps=5)[0]
    assert again == losses[:5]
    from paper_2607_10611_gb300 import fp8
    with torch.no_grad():
        batch = fp8.linear(torch.nn.functional.gelu(fp8.linear(x[:8], weights[0])), weights[1])
    assert torch.equal(example.serve(weights, x[:8]), batch)
