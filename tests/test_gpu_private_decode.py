"""examples/private_decode.py: an encrypted projection, adapters, cache and attention together, against float64."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_decoding_follows_the_plain_layer():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("private_decode", os.path.join(ROOT, "examples", "private_decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # as the layer's decryption tests: within 1e-3 of the plaintext result (the toy's encryption errors)
    assert example.run(steps=6) <= 1e-3
