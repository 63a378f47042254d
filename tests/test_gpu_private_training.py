"""examples/private_training.py: norm, encrypted projection, adapter, preference loss, their gradients and the optimiser
together, each step's gradients against float64."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_gradients_follow_the_plain_layer():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("private_training", os.path.join(ROOT, "examples", "private_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    worst, off = example.run(steps=3)
    # as the layer's decryption tests: rows within 1e-3 of the plaintext result (the toy's encryption errors), logits by as much;
    # the loss and the gradients are smooth in them (slopes of beta = 2 over 8 tokens)
    assert worst <= 2e-2 and off <= 1.6e-2
