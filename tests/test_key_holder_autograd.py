"""The key holder's binding beside autograd: its results carry no gradient, so inputs that ask for one are refused, and
what a call overwrites counts as modified.  The library's calls are stand-ins that accept everything; CPU tensors say they
are on device 0; no GPU."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32 = torch.float32


class OnDevice(torch.Tensor):
    """A CPU tensor that the binding takes for one of device 0."""

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return 0


class Library:
    def __init__(self):
        self.calls, self.status = [], 0

    def __getattr__(self, name):
        if not name.startswith("fiona_"):
            raise AttributeError(name)

        def call(*args):
            if name.endswith(("_create", "_destroy")):
                return 0
            self.calls.append(name)
            return self.status

        setattr(self, name, call)
        return call


@pytest.fixture
def binding(monkeypatch):
    spec = importlib.util.spec_from_file_location("binding_copy", os.path.join(ROOT, "paper_2609_35352_amd", "__init__.py"))
    m = importlib.util.module_from_spec(spec)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    spec.loader.exec_module(m)
    library = Library()
    monkeypatch.setattr(m, "lib", lambda: library)
    return m, library


def _tensor(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


I32, I64 = torch.int32, torch.int64
CALLS = {  # name: (its tensors, which of them it writes)
    "kv_append": (lambda: dict(k=_tensor(3, 2, 16), v=_tensor(3, 2, 16), slots=_tensor(3, dtype=I64), k_cache=_tensor(4, 8, 2, 16),
                               v_cache=_tensor(4, 8, 2, 16), positions=_tensor(3, dtype=I32), cos=_tensor(9, 8), sin=_tensor(9, 8),
                               q=_tensor(3, 4, 16), q_out=_tensor(3, 4, 16)), ("k_cache", "v_cache", "q_out")),
    "paged_attention": (lambda: dict(q=_tensor(3, 4, 16), k_cache=_tensor(4, 8, 2, 16), v_cache=_tensor(4, 8, 2, 16),
                                     page_table=_tensor(3, 4, dtype=I32), lengths=_tensor(3, dtype=I32), out=_tensor(3, 4, 16),
                                     lse=_tensor(3, 4)), ("out", "lse")),
    "adapter_linear": (lambda: dict(x=_tensor(3, 16), ids=_tensor(3, dtype=I32), A=_tensor(2, 4, 16), B=_tensor(2, 32, 4),
                                    base=_tensor(3, 32), y=_tensor(3, 32), ranks=_tensor(2, dtype=I32), scaling=_tensor(2)), ("y",)),
    "adapter_backward": (lambda: dict(x=_tensor(3, 16), ids=_tensor(3, dtype=I32), A=_tensor(2, 4, 16), B=_tensor(2, 32, 4),
                                      dy=_tensor(3, 32), dx_base=_tensor(3, 16), dx=_tensor(3, 16), dA=_tensor(2, 4, 16),
                                      dB=_tensor(2, 32, 4), ranks=_tensor(2, dtype=I32), scaling=_tensor(2)), ("dx", "dA", "dB")),
}


def _call(m, name, t):
    first = ()
    if name == "paged_attention":
        first = (m.Attention(F32, 4, 2, 16, 8, 3, 32),)
    elif name != "kv_append":
        first = (m.Adapters(F32, 2, 4, 16, 32, 3),)
    getattr(m, name)(*first, **t)


FLOATS = [(name, k) for name, (make, _) in CALLS.items() for k, v in make().items() if v.dtype is F32]


@pytest.mark.parametrize("name,which", FLOATS)
def test_tensors_that_ask_for_a_gradient_are_refused(binding, name, which):
    m, library = binding
    t = CALLS[name][0]()
    t[which].requires_grad_()
    with pytest.raises(ValueError, match="%s requires a gradient" % which):
        _call(m, name, t)
    assert library.calls == []
    with torch.no_grad():
        _call(m, name, t)
    with torch.inference_mode():
        _call(m, name, t)
    assert library.calls == ["fiona_" + name] * 2
    t[which] = t[which].detach()
    _call(m, name, t)
    assert len(library.calls) == 3


@pytest.mark.parametrize("name", list(CALLS))
def test_calls_without_gradients_go_through(binding, name):
    m, library = binding
    _call(m, name, CALLS[name][0]())
    assert library.calls == ["fiona_" + name]
