"""examples/rlvr_step.py runs, and its parts agree: the rollout's log-probabilities are the trainer's up to the
cache's rounding, and updates lower the loss."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kv,gap", [("bf16", 0.1), ("fp8", 0.5)])
def test_rlvr_step(kv, gap):
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("rlvr_step", os.path.join(ROOT, "examples", "rlvr_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history, first_gap = example.main(kv)
    # attention inputs of 8 or 3 fraction bits, logits of size 1 to 4
    assert first_gap < gap
    assert abs(history[0]["ratio"] - 1) < gap / 4 and abs(history[0]["weight"] - 1) < 1e-5
    assert history[-1]["loss"] < history[0]["loss"] and history[-1]["kl"] > history[0]["kl"]
