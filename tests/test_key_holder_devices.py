"""The key holder's binding with tensors of another device than the current one, on which its kernels would be launched:
refused before the library is called.  Stand-ins for the tensors and the library; no GPU."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Tensor:
    """What the binding asks of a contiguous device tensor."""

    is_cuda, requires_grad = True, False

    def __init__(self, dtype, shape, dev):
        self.dtype, self.shape, self.dev = dtype, torch.Size(shape), dev

    def get_device(self):
        return self.dev

    def stride(self):
        st = [1]
        for n in reversed(self.shape[1:]):
            st.append(st[-1] * n)
        return tuple(reversed(st))

    def is_contiguous(self):
        return True

    def is_inference(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Stream:
    def __init__(self, dev):
        self.device_index, self.cuda_stream = dev, 4096 + dev


class Library:
    """Accepts every call and keeps their streams."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        if not name.startswith("fiona_"):
            raise AttributeError(name)

        def call(*args):
            if not name.endswith(("_create", "_destroy")):
                self.streams.append(args[-1])
            return 0

        setattr(self, name, call)
        return call


@pytest.fixture
def binding(monkeypatch):
    """A copy of the binding of its own, on device 0, with the stand-in library."""
    spec = importlib.util.spec_from_file_location("binding_copy", os.path.join(ROOT, "paper_2609_35352_amd", "__init__.py"))
    m = importlib.util.module_from_spec(spec)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 1000 + dev, raising=False)
    monkeypatch.setattr(torch.autograd.graph, "increment_version", lambda tensors: None)   # (the stand-ins have none)
    spec.loader.exec_module(m)
    library = Library()
    monkeypatch.setattr(m, "lib", lambda: library)
    return m, library


def _calls(m, dev, **kw):
    f32, i32, i64 = torch.float32, torch.int32, torch.int64
    t = lambda dtype, *shape: Tensor(dtype, shape, dev)
    cache = lambda: t(f32, 4, 8, 2, 16)
    rows = lambda: t(f32, 3, 2, 16)
    ad = m.Adapters(f32, 2, 4, 16, 32, 3)
    yield lambda: m.kv_append(rows(), rows(), t(i64, 3), cache(), cache(), **kw)
    yield lambda: m.paged_attention(m.Attention(f32, 2, 2, 16, 8, 3, 32), rows(), cache(), cache(), t(i32, 3, 4), t(i32, 3), rows(), **kw)
    A, B = t(f32, 2, 4, 16), t(f32, 2, 32, 4)
    yield lambda: m.adapter_linear(ad, t(f32, 3, 16), t(i32, 3), A, B, None, t(f32, 3, 32), **kw)
    yield lambda: m.adapter_backward(ad, t(f32, 3, 16), t(i32, 3), A, B, t(f32, 3, 32), None, t(f32, 3, 16), t(f32, 2, 4, 16),
                                     t(f32, 2, 32, 4), **kw)


def test_tensors_of_another_device_are_refused(binding):
    m, library = binding
    for stream in (None, 77, Stream(1)):
        for call in _calls(m, 1, stream=stream):
            with pytest.raises(ValueError, match="device 1"):
                call()
    assert library.streams == []


def test_a_stream_of_another_device_is_refused(binding):
    m, library = binding
    for call in _calls(m, 0, stream=Stream(1)):
        with pytest.raises(ValueError, match="device 1"):
            call()
    assert library.streams == []


def test_calls_on_the_current_device_go_to_their_stream(binding):
    m, library = binding
    for stream in (None, 77, Stream(0)):
        for call in _calls(m, 0, stream=stream):
            call()
    assert library.streams == [1000] * 4 + [77] * 4 + [4096] * 4
