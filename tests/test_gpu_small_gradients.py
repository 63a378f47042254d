"""Optimiser steps on gradients whose squares are subnormal in 32 bits."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [3e-17, 1e-18, 1e-19])
def test_subnormal_variances_have_their_root(size):
    """32-bit states, an eps far below the gradients: the first step moves each element by about lr."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    n = 700
    g = size * (1 + torch.rand(n, generator=torch.Generator().manual_seed(1)))
    t = {k: torch.zeros(n, device=dev) for k in ("p", "m", "v")}
    opt = fiona.AdamW([t["p"]], [g.to(dev)], [t["m"]], [t["v"]], eps=1e-30, weight_decay=0.0)
    fiona.adamw_step(opt, torch.tensor([1e-3], device=dev), torch.ones(1, dtype=torch.int32, device=dev))
    m, v = 0.1 * g.double(), 1e-3 * g.double() ** 2
    lr = float(torch.tensor(1e-3))
    step = m / (1 - 0.9) / ((v / (1 - 0.999)).sqrt() + 1e-30)
    # v is a sum of two products, g^2 one more (each may be subnormal: off by 2^-150 besides E of itself); its root by half of
    # that, and 24 E for the rest as in ref.adamw
    dv = 6 * ref.E + (2.0 ** -150 * (2 + 1e-3)) / v
    bound = 2 * lr * step * (dv / 2 + 24 * ref.E)
    assert bool((bound < 0.2 * lr).all())
    ref.assert_close(t["p"], -lr * step, bound, "parameters")
