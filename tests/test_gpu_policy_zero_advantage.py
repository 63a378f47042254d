"""Tokens without advantage whose ratio passes what 32 bits hold."""
import pytest

torch = pytest.importorskip("torch")
import test_gpu_token_loss as tl  # noqa: E402
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,V", [(6, 500), (6, 3), (3, 50021)])
@pytest.mark.parametrize("gradient", [True, False])
@pytest.mark.parametrize("kl", [0.0, 0.05])
def test_no_advantage_is_no_loss(n, V, gradient, kl):
    dev = tl._dev()
    c = tl._tokens(n, V, torch.float32, seed=V, masked=0.0)
    c["advantages"][::2] = 0.0
    c["old"][0], c["old"][2] = -200.0, -95.0         # exp(l - old) beyond 2^128
    got = tl._policy(c, dev, gradient=gradient, kl=kl)
    tl._check_policy(c, got, kl=kl)
    if kl == 0:
        assert float(got[0][0]) == 0 and (not gradient or not got[2][0].any())
