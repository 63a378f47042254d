"""What the key holder's calls overwrite counts as modified, so that autograd refuses a backward pass over values that
are gone (the stand-ins of test_key_holder_autograd; no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from test_key_holder_autograd import CALLS, _call, _tensor, binding  # noqa: E402,F401


@pytest.mark.parametrize("name", list(CALLS))
def test_outputs_count_as_modified_and_inputs_do_not(binding, name):  # noqa: F811
    m, library = binding
    t = CALLS[name][0]()
    before = {k: v._version for k, v in t.items()}
    _call(m, name, t)
    for k, v in t.items():
        assert (v._version > before[k]) == (k in CALLS[name][1]), k
    after = {k: v._version for k, v in t.items()}
    library.status = -1                 # a refused call writes nothing
    with pytest.raises(m.FionaError):
        _call(m, name, t)
    assert {k: v._version for k, v in t.items()} == after


@pytest.mark.parametrize("name,out,source", [("kv_append", "q_out", "q"), ("adapter_linear", "y", "base"),
                                             ("adapter_backward", "dx", "dx_base")])
def test_a_saved_tensor_overwritten_in_place_is_noticed(binding, name, out, source):  # noqa: F811
    m, _ = binding
    t = CALLS[name][0]()
    w = torch.ones(t[source].shape, requires_grad=True)
    loss = (w * t[source].as_subclass(torch.Tensor)).sum()       # saves the source for w's gradient
    t[out] = t[source]
    _call(m, name, t)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inference_tensors_are_taken(binding):  # noqa: F811
    m, library = binding
    with torch.inference_mode():
        t = CALLS["adapter_linear"][0]()
        _call(m, "adapter_linear", t)
    _call(m, "adapter_linear", dict(t, x=_tensor(3, 16)))
    assert len(library.calls) == 2
