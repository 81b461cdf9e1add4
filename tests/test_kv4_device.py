"""Which device the binding of the 4-bit cache makes its calls on (CPU: devices, streams and the library are stood in for)."""
import contextlib
import types

import pytest
import torch

import paper_2312_04916_amd.kv4 as kv4


@pytest.fixture
def cache(monkeypatch):
    """A cache on cuda:1, device 0 being the current one; what the library is called with, and the device that is current then."""
    current, calls = [0], []

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    def entry(name):
        def fn(handle, *args):
            calls.append((name, current[0], args[-1]))
            return 0
        return fn

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda where=None: calls.append(("synchronize", where, None)))
    monkeypatch.setattr(kv4, "_current_device", lambda: current[0], raising=False)
    monkeypatch.setattr(kv4, "_current_stream", lambda index: 0, raising=False)
    monkeypatch.setattr(kv4, "lib", lambda: types.SimpleNamespace(ee_kv4_free=lambda h: 0))
    monkeypatch.setattr(kv4.Kv4Cache, "_lengths", lambda self, t, n, what: 256)
    monkeypatch.setattr(kv4.Kv4Cache, "_vectors", lambda self, t, heads, rows, what: (256, 1, 1))
    monkeypatch.setattr(kv4.Kv4Cache, "_slot_ptr", lambda self, slots, rows: 256)
    monkeypatch.setattr(kv4.Kv4Cache, "_empty", lambda self, stream, *shape, dtype: torch.empty(shape, dtype=dtype))
    c = kv4.Kv4Cache.__new__(kv4.Kv4Cache)
    c.h, c.device, c._index, c.dtype, c.n_rows = 1, torch.device("cuda:1"), 1, torch.bfloat16, 2
    c._heads, c._kv_heads, c._head_dim = 4, 2, 64
    c._plan, c._append, c._read, c._attend = (entry(n) for n in ("plan", "append", "read", "attend"))
    yield c, calls, current
    c.h = 0


def each_call(c, stream=None):
    i, x, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 64), torch.zeros(2, dtype=torch.int64)
    return [lambda: c.plan(i, i, i, 2, stream=stream), lambda: c.append(0, x, x, stream=stream), lambda: c.read(0, slots, stream=stream),
            lambda: c.attend(0, x, stream=stream)]


def test_calls_go_to_the_cache_s_device(cache):
    c, calls, current = cache
    for now in (0, 1, 2):
        current[0] = now
        calls.clear()
        for call in each_call(c):
            call()
        assert calls == [(n, 1, 0) for n in ("plan", "append", "read", "attend")]
        assert current[0] == now
    calls.clear()
    c.close()
    assert calls == [("synchronize", torch.device("cuda:1"), None)]


def test_streams_of_other_devices_are_refused(cache):
    c, calls, _ = cache
    for call in each_call(c, types.SimpleNamespace(device_index=0, cuda_stream=7)):
        with pytest.raises(ValueError, match="stream of device 0"):
            call()
    assert calls == []
