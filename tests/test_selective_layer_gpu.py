"""The layer of examples/selective_layer.py: gradients reach every parameter and the
loss falls; prompts in one packed call followed by single tokens give what one call
over all tokens gives."""
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
    import selective_layer

    torch.manual_seed(0)
    return selective_layer


def test_training_reaches_every_parameter(example):
    import torch

    print("selective layer: training", flush=True)
    layer = example.SelectiveLayer(model=128, inner=256)
    losses = example.train(layer, steps=12, B=2, T=100)
    assert losses[-1] < losses[0], losses
    for name, p in layer.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any(), name


def test_steps_continue_a_packed_prompt(example):
    print("selective layer: serving", flush=True)
    layer = example.SelectiveLayer(model=128, inner=256)
    got, want = example.serve(layer, lens=(70, 1, 133, 2), new=4)
    # bf16 throughout: the same values rounded at the same places, but torch's products may
    # split their sums otherwise for other row counts: a unit in the last place (2^-8) of some
    # intermediate, four products deep
    err = (got - want).float().abs().max().item()
    assert err <= 2.0 ** -5 * want.float().abs().max().item(), err
