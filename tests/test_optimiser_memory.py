"""An optimiser's tensors are other tensors' memory, kept whatever becomes of those (the stand-ins of
test_key_holder_autograd; no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from test_key_holder_autograd import OnDevice, _tensor, binding  # noqa: E402,F401

F16, F32 = torch.float16, torch.float32
KEYS = ("params", "grads", "m", "v", "masters")


@pytest.mark.parametrize("which", KEYS)
@pytest.mark.parametrize("asks", [False, True])
def test_memory_is_kept_where_tensors_ask_for_a_gradient(binding, which, asks):  # noqa: F811
    m, _ = binding
    t = {k: [_tensor(5, dtype=F16 if k in ("params", "grads") else F32) for _ in range(2)] for k in KEYS}
    t[which][1].requires_grad_(asks)
    with torch.no_grad():                       # (taken there, as every call takes them)
        opt = m.AdamW(**t)
    at = {k: [x.data_ptr() for x in xs] for k, xs in t.items()}
    for xs in t.values():
        for x in xs:
            x.data = torch.zeros(3, dtype=x.dtype).as_subclass(OnDevice)
    assert {k: [x.data_ptr() for x in xs] for k, xs in opt._tensors.items()} == at
    assert all(x.numel() == 5 and not x.requires_grad for xs in opt._tensors.values() for x in xs)


@pytest.mark.parametrize("which", [k for k in KEYS if k != "params"])
def test_tensors_that_ask_for_a_gradient_are_refused_in_grad_mode(binding, which):  # noqa: F811
    m, _ = binding
    t = {k: [_tensor(5, dtype=F16 if k in ("params", "grads") else F32) for _ in range(2)] for k in KEYS}
    t[which][1].requires_grad_()
    with pytest.raises(ValueError, match=r"%s\[1\] requires a gradient" % which):
        m.AdamW(**t)
