"""The example that runs the operators on logits together with the quantized layer."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "distill_output_layer.py")
    spec = importlib.util.spec_from_file_location("distill_output_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("vocab", [1000, 4104])
def test_distillation_improves_the_student(example, vocab):
    losses, before, after = example.run(tokens=256, vocab=vocab, hidden=256, steps=12)
    assert all(loss == loss and loss > 0 for loss in losses)
    assert after[0] < before[0]                  # on tokens that were not trained on


def test_calls_and_autograd_agree(example):
    """Both run the same products and the same loss; bf16 gradients scaled by 1/T before or after their rounding and two
    AdamW implementations: a step of AdamW is at most lr per scale either way, so losses differ in their third digit at most."""
    args = dict(tokens=256, vocab=1000, hidden=256, steps=6)
    calls, nodes = example.run(**args)[0], example.run(use_autograd=True, **args)[0]
    assert calls[0] == pytest.approx(nodes[0], rel=1e-5)
    for a, b in zip(calls, nodes):
        assert a == pytest.approx(b, rel=1e-2)
