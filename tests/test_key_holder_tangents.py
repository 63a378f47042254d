"""Tensors that carry a forward-mode tangent are refused by every call of the key holder's (the stand-ins of
test_key_holder_autograd; no GPU)."""
import pytest

torch = pytest.importorskip("torch")
import test_key_holder_autograd as key_holder  # noqa: E402
import test_training_binding as training  # noqa: E402
from test_key_holder_autograd import OnDevice, _tensor, binding  # noqa: E402,F401

fwd = torch.autograd.forward_ad
F32 = torch.float32
FLOATS = [(part, name, k) for part in (key_holder, training) for name, (make, _) in part.CALLS.items() for k, v in make().items()
          if v.dtype is F32]


@pytest.mark.parametrize("part,name,which", FLOATS)
def test_tangents_are_refused(binding, part, name, which):  # noqa: F811
    m, library = binding
    t = part.CALLS[name][0]()
    with fwd.dual_level():
        plain = t[which]
        t[which] = fwd.make_dual(plain, torch.ones_like(plain)).as_subclass(OnDevice)
        assert fwd.unpack_dual(t[which]).tangent is not None
        for mode in (torch.enable_grad, torch.no_grad):
            with mode(), pytest.raises(ValueError, match="%s carries a tangent" % which):
                part._call(m, name, t)
        assert library.calls == []
        t[which] = t[which].detach()
        part._call(m, name, t)
        t[which] = plain
        part._call(m, name, t)
    part._call(m, name, t)
    assert library.calls == ["fiona_" + name] * 3


@pytest.mark.parametrize("which", ["params", "grads", "m", "v", "masters"])
def test_an_optimiser_refuses_them(binding, which):  # noqa: F811
    m, _ = binding
    t = {k: [_tensor(5, dtype=torch.float16 if k in ("params", "grads") else F32) for _ in range(2)] for k in ("params", "grads", "m", "v", "masters")}
    with fwd.dual_level():
        x = t[which][1]
        t[which][1] = fwd.make_dual(x, torch.ones_like(x)).as_subclass(OnDevice)
        with torch.no_grad(), pytest.raises(ValueError, match=r"%s\[1\] carries a tangent" % which):
            m.AdamW(**t)
        t[which][1] = x
        m.AdamW(**t)
