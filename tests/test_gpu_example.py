"""The example that trains and serves a hybrid stack with the scan, the gated
linear recurrence, the feed-forward block and the 8-bit AdamW step: it learns,
and token by token it gives what the whole sequence gives."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("hybrid_stack", os.path.join(ROOT, "examples", "hybrid_stack.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_trains_and_serves(example):
    f32, low, losses = example.train(steps=60, tell=lambda s: print(s, flush=True))
    assert all(v == v for v in losses)
    # the target's variance is 0.31^2 / (1 - 0.95^2) = 0.99: what a stack without memory leaves
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0] and losses[-1] < 0.5
    whole, steps, want = example.serve(f32, low)
    # bf16 activations at about twenty roundings, of a result of size one
    assert torch.isfinite(steps).all()
    assert (whole - steps).abs().max().item() <= 20 * 2.0 ** -8 * whole.abs().max().item()
    assert torch.nn.functional.mse_loss(steps, want).item() < 0.6
