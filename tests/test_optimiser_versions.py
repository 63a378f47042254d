"""A step counts each version counter that its tensors have once (the stand-ins of test_key_holder_autograd; no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from test_key_holder_autograd import OnDevice, _tensor, binding  # noqa: E402,F401


class _Views:
    """Tensors that lie in one, as an optimiser's often do."""

    def __init__(self, asks=False):
        self.store = torch.zeros(8 * 10).as_subclass(OnDevice).requires_grad_(asks)
        with torch.no_grad():
            self.views = list(self.store.view(8, 10).unbind())


@pytest.mark.parametrize("asks", [False, True])
def test_views_of_one_tensor_count_once(binding, asks):  # noqa: F811
    m, _ = binding
    t = {k: _Views(asks and k == "params") for k in ("params", "grads", "m", "v")}
    opt = m.AdamW(**{k: x.views for k, x in t.items()})
    assert len(opt._written) == 3
    before = {k: (x.store._version, [y._version for y in x.views]) for k, x in t.items()}
    m.adamw_step(opt, _tensor(1), _tensor(1, dtype=torch.int32))
    for k, x in t.items():
        written = int(k != "grads")
        assert x.store._version == before[k][0] + written, k
        assert [y._version for y in x.views] == [b + written for b in before[k][1]], k


def test_views_and_tensors_of_their_own(binding):  # noqa: F811
    m, _ = binding
    t = _Views()
    own = [_tensor(10) for _ in range(8)]
    zeros = lambda: [_tensor(10) for _ in range(8)]
    opt = m.AdamW(t.views[:4] + own[4:], zeros(), zeros(), zeros())
    assert len(opt._written) == 1 + 4 + 8 + 8
    m.adamw_step(opt, _tensor(1), _tensor(1, dtype=torch.int32))
    assert t.store._version == 1 and [x._version for x in own] == [0] * 4 + [1] * 4
