"""The training step's binding: tensors that ask for a gradient and tensors or streams of another device are refused, and
what a call overwrites counts as modified (the stand-ins of test_key_holder_autograd; no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from test_key_holder_autograd import OnDevice, _tensor, binding  # noqa: E402,F401

F32, I32 = torch.float32, torch.int32
CALLS = {  # name: (its tensors, which of them it writes)
    "layer_norm": (lambda: dict(x=_tensor(3, 16), weight=_tensor(16), bias=_tensor(16), y=_tensor(3, 16), residual=_tensor(3, 16),
                                total=_tensor(3, 16), mean=_tensor(3), rstd=_tensor(3)), ("y", "total", "mean", "rstd")),
    "layer_norm_backward": (lambda: dict(dy=_tensor(3, 16), x=_tensor(3, 16), weight=_tensor(16), mean=_tensor(3), rstd=_tensor(3),
                                         dx_base=_tensor(3, 16), dx=_tensor(3, 16), dweight=_tensor(16), dbias=_tensor(16)),
                            ("dx", "dweight", "dbias")),
    "preference_loss": (lambda: dict(logits=_tensor(4, 9), targets=_tensor(4, dtype=I32), offsets=_tensor(3, dtype=I32),
                                     reference=_tensor(2), loss=_tensor(1), logps=_tensor(2), dlogits=_tensor(4, 9), weights=_tensor(1)),
                        ("loss", "logps", "dlogits")),
    "policy_loss": (lambda: dict(logits=_tensor(4, 9), targets=_tensor(4, dtype=I32), old=_tensor(4), advantages=_tensor(4),
                                 loss=_tensor(4), logps=_tensor(4), dlogits=_tensor(4, 9), reference=_tensor(4), weights=_tensor(4)),
                    ("loss", "logps", "dlogits")),
    "adamw_step": (lambda: dict(lr=_tensor(1), step=_tensor(1, dtype=I32), grad_scale=_tensor(1)), ()),
}


def _handle(m, name):
    if name == "layer_norm":
        return ()
    if name == "layer_norm_backward":
        return (m.LayerNorm(F32, 16, 3),)
    if name == "adamw_step":
        return (m.AdamW([_tensor(5)], [_tensor(5)], [_tensor(5)], [_tensor(5)]),)
    return (m.TokenLoss(F32, 9, 4, 1),)


def _call(m, name, t, **kw):
    getattr(m, name)(*_handle(m, name), **t, **kw)


@pytest.mark.parametrize("name,which", [(name, k) for name, (make, _) in CALLS.items() for k, v in make().items() if v.dtype is F32])
def test_tensors_that_ask_for_a_gradient_are_refused(binding, name, which):  # noqa: F811
    m, library = binding
    t = CALLS[name][0]()
    t[which].requires_grad_()
    with pytest.raises(ValueError, match="%s requires a gradient" % which):
        _call(m, name, t)
    assert library.calls == []
    with torch.no_grad():
        _call(m, name, t)
    t[which] = t[which].detach()
    _call(m, name, t)
    assert library.calls == ["fiona_" + name] * 2


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


def test_a_step_counts_as_modifying_the_optimisers_tensors(binding):  # noqa: F811
    m, _ = binding
    store = torch.zeros(64)
    view = store[3:8].as_subclass(OnDevice)
    w = _tensor(5).requires_grad_()
    t = dict(params=[w, view], grads=[_tensor(5), _tensor(5)], m=[_tensor(5), _tensor(5)], v=[_tensor(5), _tensor(5)])
    opt = m.AdamW(**t)
    before = {k: [x._version for x in v] for k, v in t.items()}
    m.adamw_step(opt, _tensor(1), _tensor(1, dtype=I32))
    for k, v in t.items():
        assert [x._version > b for x, b in zip(v, before[k])] == [k != "grads"] * 2, k
    for k in ("grads", "m", "v"):
        with pytest.raises(ValueError, match="requires a gradient"):
            m.AdamW(**dict(t, **{k: [t[k][0], _tensor(5).requires_grad_()]}))


def test_devices_and_streams(binding):  # noqa: F811
    m, library = binding

    class Stream:
        device_index, cuda_stream = 1, 4097

    for name, (make, _) in CALLS.items():
        with pytest.raises(ValueError, match="device 1"):
            _call(m, name, make(), stream=Stream())
    m._device_now[0] = lambda: 1
    for name, (make, _) in CALLS.items():
        with pytest.raises(ValueError, match="device"):
            _call(m, name, make())
    assert library.calls == []
