"""The blocks of examples/decay_blocks.py: gradients reach every parameter; prompts in one
packed call followed by single tokens give what one call over all tokens gives."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def example():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import decay_blocks

    torch.manual_seed(0)
    return decay_blocks


def test_training_reaches_every_parameter(example):
    import torch

    model = example.DecayBlocks(model=128, layers=2, heads=4, dk=48, dv=40)
    example.train(model, steps=3, B=2, T=100)
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any(), name


def test_steps_continue_a_packed_prompt(example):
    model = example.DecayBlocks(model=128, layers=2, heads=4, dk=48, dv=40)
    got, want = example.serve(model, lens=(70, 1, 133, 2), new=4)
    # bf16 throughout, by other routes (a step multiplies in fp32 what a chunk rounds to
    # bf16): half a step, 2^-8, of some intermediate in each of the two layers' four products
    # and roundings, and the norms keep relative errors
    err = (got - want).float().abs().max().item()
    assert err <= 2.0 ** -5 * want.float().abs().max().item(), err
