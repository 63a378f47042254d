"""The key holder's binding used first by two threads: whenever one of them gets a type's code, all that a call takes from
the module's tables is there.  The second thread is played at every line of the first one's set-up; no GPU."""
import ctypes
import importlib.util
import os
import sys
import threading
import time

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "paper_2609_35352_amd", "__init__.py")


def _copy():
    spec = importlib.util.spec_from_file_location("binding_copy", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _ready(m):
    """What kv_append and the others look up once they have a type's code."""
    assert m._type_code(torch.bfloat16) == 2
    assert m._INT[4] is torch.int32 and m._INT[8] is torch.int64 and m._INT["f32"] is torch.float32
    assert callable(m._raw_stream[0]) and callable(m._device_now[0]) and callable(m._modified[0])
    L = m.lib()
    assert all(getattr(L, name).argtypes is not None for name in (
        "fiona_kv_append", "fiona_attention_create", "fiona_paged_attention", "fiona_adapters_create", "fiona_adapter_linear",
        "fiona_adapter_backward", "fiona_attention_destroy", "fiona_adapters_destroy"))


def test_a_second_thread_at_every_line_of_the_set_up():
    if not os.path.exists(_copy().LIB_PATH):
        pytest.fail("libfiona.so is not built (run __graft_entry__.build())")
    lines = 0
    for stop in range(10000):
        m = _copy()
        seen, failed = [0], []

        def trace(frame, event, arg):
            if frame.f_code.co_name != "_lm_lib" or frame.f_code.co_filename != PATH:
                return None

            def line(frame, event, arg):
                if event == "line":
                    if seen[0] == stop:
                        sys.settrace(None)
                        try:
                            _ready(m)
                        except Exception as e:   # (an exception here would only end the trace)
                            failed.append("line %d: %r" % (frame.f_lineno, e))
                    seen[0] += 1
                return line

            return line

        sys.settrace(trace)
        try:
            m._lm_lib()
        finally:
            sys.settrace(None)
        assert not failed, failed
        _ready(m)
        if seen[0] <= stop:
            break
        lines += 1
    assert lines > 8


def test_two_threads_load_one_library(monkeypatch):
    """Two loads would leave the functions of one without their argument types (a stream's handle cut to 32 bits)."""
    m = _copy()
    if not os.path.exists(m.LIB_PATH):
        pytest.fail("libfiona.so is not built (run __graft_entry__.build())")
    load, loads = ctypes.CDLL, []

    def slow(path, *args, **kw):
        loads.append(path)
        time.sleep(0.3)
        return load(path, *args, **kw)

    monkeypatch.setattr(ctypes, "CDLL", slow)
    failed = []

    def use():
        try:
            _ready(m)
        except Exception as e:
            failed.append(repr(e))

    threads = [threading.Thread(target=use) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and loads == [m.LIB_PATH]
    _ready(m)
