"""examples/mlp_block.py: the operators together as a training step of an MLP block."""
import importlib.util
import os

import pytest
import torch

from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("mlp_block", os.path.join(ROOT, "examples", "mlp_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("tokens,d_model,d_ffn", [(256, 512, 1024), (1040, 528, 2064)])
def test_a_step_is_near_the_block_in_64_bits(example, tokens, d_model, d_ffn):
    """A block's largest magnitude is 6 of E2M1's steps: rounding is off by some 0.1 of a value (the step 0.5 .. 2 over 2 sqrt(3) against values of 0.5 to 6), so
    each product's operands bring 0.1 each and its result sqrt(2) 0.1; squared ReLU doubles what reaches it, and a gradient passes two products.  y is mostly
    its residual.  A wrong formula (a missing factor, bias or derivative) is off by 0.5 and more in what it touches."""
    errors = example.main(tokens, d_model, d_ffn)
    assert errors["y"] < 0.2
    for name in ("dx", "gamma", "w1", "b1", "w2"):
        assert errors[name] < 0.4, (name, errors)
    assert errors["b2"] < 1e-5      # a sum of dy itself


def test_micro_batches_accumulate_and_a_step_repeats_bit_for_bit(example):
    block = example.MlpBlock(512, 1024)
    x, r, dy = (torch.randn(256, 512, device="cuda").bfloat16() for _ in range(3))
    y, saved = block.forward(x, r)
    dx = block.backward(dy, saved, 3)
    once = {k: v.clone() for k, v in block.grads.items()}
    y2, saved = block.forward(x, r)
    dx2 = block.backward(dy, saved, 3)
    assert torch.equal(y, y2) and torch.equal(dx, dx2)
    for name, g in block.grads.items():
        assert torch.equal(g, 2 * once[name]), name      # a sum and itself: exact


def test_the_norms_output_can_be_made_again_from_its_checkpoint(example):
    """Instead of the 4-bit copy: n from the 8 bits and gamma, quantized again."""
    block = example.MlpBlock(512, 1024)
    x, r = (torch.randn(256, 512, device="cuda").bfloat16() for _ in range(2))
    norm = nv.nvfp4_rmsnorm_forward(x, block.gamma, residual=r, checkpoint=True)
    again = nv.nvfp4_checkpoint_load(norm.checkpoint, col_scale=block.gamma)
    off = (again.float() - norm.y.float()).abs()
    assert bool((off <= (2.0 ** -4 + 2.0 ** -7) * norm.y.float().abs() + 2.0 ** -10 * 1.5).all())
