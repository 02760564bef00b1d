"""The example block trains and generates: norms, projections, the gated pair and the cell together, forward, backward and token by
token, and its backward pass against differences."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("residual_block", os.path.join(ROOT, "examples", "residual_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss_and_both_ways_agree(example):
    losses, worst = example.run(tokens=192, heads=2, dqk=64, dhv=64, steps=12)
    assert losses[-1] < 0.9 * losses[0], losses
    # every tensor on the way is rounded to bf16 (2^-8 of its value, some ten of them one after another) by either way, and
    # they share none of the cell's kernels
    assert worst <= 2 * 10 * 2.0 ** -8, worst


def test_odd_sizes_run(example):
    block = example.Block(3, 64, 64)
    x = torch.randn((1, 77, block.D), device="cuda").to(torch.bfloat16)
    out, saved = block.forward(x)
    dx, grads = block.backward(saved, torch.ones_like(out))
    assert dx.shape == x.shape and all(bool(torch.isfinite(g).all()) for g in grads.values())
    assert grads["in"].shape == block.w["in"].shape and grads["down"].shape == block.w["down"].shape
