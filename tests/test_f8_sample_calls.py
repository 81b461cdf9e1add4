"""Products with 8-bit weights and choosing tokens: sizes and refusals that need no GPU, and the device that the binding calls on (CPU:
devices, streams and the library are stood in for)."""
import contextlib
import ctypes as C
import types

import numpy as np
import pytest
import torch

import paper_2312_04916_amd as ee
import paper_2312_04916_amd.f8 as f8
import paper_2312_04916_amd.sampling as sampling

F32, BF16 = ee.EE_F32, ee.EE_BF16
GOOD, ARG, CONFIG, NOMEM = 0, -7, -1, -2


def test_sizes():
    L, b = ee.lib(), C.c_size_t()
    for n, k, pair in ((1, 1, 0), (16, 128, 0), (17, 129, 1), (50304, 4096, 0), (11008, 4096, 1), (1 << 22, 1 << 18, 1)):
        assert L.ee_f8_bytes(n, k, pair, C.byref(b)) == GOOD
        tiles, steps = -(-n // 16) * (1 + pair), -(-k // 128)
        assert tiles * steps * 2049 <= b.value <= tiles * steps * 2049 + 256
    for n, k in ((0, 1), (1, 0), (-1, 5), ((1 << 22) + 1, 1), (1, (1 << 18) + 1)):
        assert L.ee_f8_bytes(n, k, 0, C.byref(b)) == CONFIG
        assert L.ee_f8_matmul_bytes(1, n, k, 0, BF16, C.byref(b)) == CONFIG
    assert L.ee_f8_bytes(1, 1, 0, None) == ARG
    assert L.ee_f8_matmul_bytes(0, 64, 64, 0, F32, C.byref(b)) == GOOD
    assert L.ee_f8_matmul_bytes(1 << 20, 64, 64, 0, F32, C.byref(b)) == GOOD
    for m in (-1, (1 << 20) + 1):
        assert L.ee_f8_matmul_bytes(m, 64, 64, 0, F32, C.byref(b)) == ARG
    assert L.ee_f8_matmul_bytes(1, 64, 64, 0, 2, C.byref(b)) == CONFIG


def test_pack_refusals():
    L, big = ee.lib(), 1 << 40
    pack = lambda n=64, k=64, pair=0, dt=BF16, w=4096, ws=64, up=None, us=0, p=1 << 20, size=big: L.ee_f8_pack(n, k, pair, dt, w, ws, up, us, p, size, None)  # noqa: E731
    for bad, code in ((dict(n=0), CONFIG), (dict(dt=2), CONFIG), (dict(w=None), ARG), (dict(p=None), ARG), (dict(p=(1 << 20) + 16), ARG), (dict(w=4097), ARG),
                      (dict(dt=F32, w=4098), ARG), (dict(pair=1), ARG), (dict(up=8192), ARG), (dict(size=100), NOMEM), (dict(w=(1 << 20) + 64), ARG),
                      (dict(pair=1, up=(1 << 20) - 64, us=64), ARG)):
        assert pack(**bad) == code, bad
    un = lambda up=0, pair=0, p=1 << 20, dt=BF16, w=4096: L.ee_f8_unpack(64, 64, pair, up, p, dt, w, None)  # noqa: E731
    for bad, code in ((dict(up=1), ARG), (dict(p=None), ARG), (dict(w=None), ARG), (dict(dt=5), CONFIG), (dict(w=4097), ARG), (dict(w=(1 << 20) + 128), ARG)):
        assert un(**bad) == code, bad


def test_matmul_refusals():
    L, big = ee.lib(), 1 << 40
    M = 1 << 24

    def mm(m=300, n=64, k=64, pair=0, w=1 * M, xd=BF16, x=2 * M, xr=64, yd=BF16, y=3 * M, yr=64, add=None, ar=0, work=4 * M, size=big):
        return L.ee_f8_matmul(m, n, k, pair, w, xd, x, xr, yd, y, yr, add, ar, work, size, None)

    for bad, code in ((dict(m=-1), ARG), (dict(m=(1 << 20) + 1), ARG), (dict(n=0), CONFIG), (dict(k=1 << 19), CONFIG), (dict(xd=3), CONFIG), (dict(yd=3), CONFIG),
                      (dict(w=None), ARG), (dict(w=M + 128), ARG), (dict(x=None), ARG), (dict(x=2 * M + 1), ARG), (dict(xd=F32, x=2 * M + 2), ARG), (dict(y=None), ARG),
                      (dict(y=3 * M + 1), ARG), (dict(yd=F32, y=3 * M + 2), ARG), (dict(add=5 * M + 1, ar=64), ARG), (dict(yr=63), ARG), (dict(yr=0), ARG), (dict(yr=-63), ARG),
                      (dict(y=2 * M), ARG), (dict(y=2 * M + 300 * 128 - 2), ARG), (dict(y=1 * M), ARG),
                      # added rows are the result's own, or apart from them
                      (dict(add=3 * M + 2, ar=64), ARG), (dict(add=3 * M, ar=128), ARG), (dict(add=3 * M - 64, ar=64), ARG),
                      # a pass over 300 rows needs its workspace
                      (dict(size=100), NOMEM), (dict(work=None), ARG), (dict(work=4 * M + 16), ARG), (dict(work=2 * M), ARG), (dict(work=3 * M), ARG), (dict(work=1 * M), ARG),
                      (dict(add=4 * M, ar=64), ARG)):
        assert mm(**bad) == code, bad
    assert mm(m=0) == GOOD and mm(m=0, x=None, y=None, w=None) == GOOD


def test_sample_refusals():
    L, b = ee.lib(), C.c_size_t()
    assert L.ee_sample_bytes(3, 1, C.byref(b)) == GOOD and b.value >= 3 * 76
    assert L.ee_sample_bytes(0, 1 << 18, C.byref(b)) == GOOD and b.value == 0
    assert L.ee_sample_bytes(1, 0, C.byref(b)) == CONFIG and L.ee_sample_bytes(1, (1 << 18) + 1, C.byref(b)) == CONFIG
    assert L.ee_sample_bytes(-1, 5, C.byref(b)) == ARG and L.ee_sample_bytes(1, 5, None) == ARG
    M = 1 << 20

    def sample(rows=4, vocab=100, dt=F32, z=M, zr=100, u=2 * M, tp=None, kp=None, pp=None, mp=None, t=1.0, k=0, p=1.0, m=0.0, token=3 * M, lp=None, cf=None, work=6 * M, size=1 << 30):
        return L.ee_sample(rows, vocab, dt, z, zr, u, tp, kp, pp, mp, t, k, p, m, token, lp, cf, work, size, None)

    nan, inf = float("nan"), float("inf")
    for bad, code in ((dict(rows=-1), ARG), (dict(rows=(1 << 20) + 1), ARG), (dict(vocab=0), CONFIG), (dict(vocab=(1 << 18) + 1), CONFIG), (dict(dt=2), CONFIG),
                      (dict(z=None), ARG), (dict(z=M + 2), ARG), (dict(u=None), ARG), (dict(u=2 * M + 2), ARG), (dict(token=None), ARG), (dict(token=3 * M + 1), ARG),
                      (dict(tp=M + 1), ARG), (dict(lp=M * 5 + 2), ARG), (dict(t=-1.0), ARG), (dict(t=nan), ARG), (dict(t=inf), ARG), (dict(k=-1), ARG), (dict(p=-0.1), ARG),
                      (dict(p=1.5), ARG), (dict(p=nan), ARG), (dict(m=-0.1), ARG), (dict(m=2.0), ARG), (dict(m=nan), ARG),
                      # results apart from what is read, and from one another
                      (dict(token=M + 1596), ARG), (dict(token=2 * M), ARG), (dict(lp=3 * M + 12), ARG), (dict(cf=3 * M), ARG), (dict(lp=4 * M, cf=4 * M), ARG),
                      (dict(tp=4 * M, lp=4 * M), ARG),
                      (dict(work=None), ARG), (dict(work=6 * M + 16), ARG), (dict(size=100), NOMEM), (dict(work=M), ARG), (dict(work=3 * M), ARG),
                      (dict(work=2 * M), ARG), (dict(cf=6 * M), ARG)):
        assert sample(**bad) == code, bad
    assert sample(rows=0) == GOOD and sample(rows=0, z=None, u=None, token=None) == GOOD


# ---------------------------------------------------------------- the binding

class Fake:
    """A tensor on cuda:1, as far as the binding looks."""

    def __init__(self, t, index=1):
        self.t, self.index = t, index

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 4096

    def record_stream(self, stream):
        pass


@pytest.fixture
def machine(monkeypatch):
    current, calls = [0], []

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    monkeypatch.setattr(torch.cuda, "device", device)
    for module in (f8, sampling):
        monkeypatch.setattr(module, "_current_device", lambda: current[0])
    monkeypatch.setattr(sampling, "_raw_stream", lambda stream, index: _stream(stream, index))
    monkeypatch.setattr(f8, "_raw_stream", lambda stream, index: _stream(stream, index))

    def _stream(stream, index):
        if stream is not None and stream.device_index != index:
            raise ValueError(f"stream of device {stream.device_index}, expected cuda:{index}")
        return 0 if stream is None else stream.cuda_stream

    def entry(name):
        def fn(*args):
            calls.append((name, current[0], args[-1]))
            return 0
        return fn

    return current, calls, entry


def weight(entry):
    w = f8.F8Weight.__new__(f8.F8Weight)
    w.n, w.k, w.pair, w.device, w._index = 8, 16, False, torch.device("cuda:1"), 1
    w._matmul, w._address, w._work = entry("matmul"), 256, {(2, BF16): 0}
    w._empty = lambda stream, *shape, dtype: torch.empty(shape, dtype=dtype)
    return w


def test_products_go_to_the_weight_s_device(machine):
    current, calls, entry = machine
    w, x = weight(entry), Fake(torch.zeros(2, 16, dtype=torch.bfloat16))
    for now in (0, 1, 2):
        current[0] = now
        w.matmul(x)
        assert calls[-1] == ("matmul", 1, 0) and current[0] == now
    calls.clear()
    with pytest.raises(ValueError, match="stream of device 0"):
        w.matmul(x, stream=types.SimpleNamespace(device_index=0, cuda_stream=7))
    bf = torch.bfloat16
    for bad in (dict(x=Fake(torch.zeros(2, 16, dtype=bf), 0)), dict(x=Fake(torch.zeros(2, 15, dtype=bf))), dict(x=Fake(torch.zeros(2, 16, dtype=torch.float16))),
                dict(x=Fake(torch.zeros(16, 2, dtype=bf).T)), dict(x=Fake(torch.zeros(16, dtype=bf))), dict(dtype=torch.float16), dict(add=Fake(torch.zeros(2, 8))),
                dict(add=Fake(torch.zeros(2, 9, dtype=bf))), dict(add=Fake(torch.zeros(1, 8, dtype=bf))), dict(add=Fake(torch.zeros(2, 8, dtype=bf), 0)),
                dict(out=Fake(torch.zeros(2, 9, dtype=bf))), dict(out=Fake(torch.zeros(3, 8, dtype=bf))), dict(out=Fake(torch.zeros(2, 8)), dtype=bf)):
        with pytest.raises(ValueError):
            w.matmul(**{"x": x, **bad})
    assert calls == []


def test_samples_go_to_the_logits_device(machine, monkeypatch):
    current, calls, entry = machine
    monkeypatch.setattr(sampling, "_fn", entry("sample"))
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    z, u = Fake(torch.zeros(2, 16)), Fake(torch.zeros(2))
    for now in (0, 1, 2):
        current[0] = now
        sampling.sample(z, u)
        assert calls[-1] == ("sample", 1, 0) and current[0] == now
    calls.clear()
    with pytest.raises(ValueError, match="stream of device 0"):
        sampling.sample(z, u, out=Fake(torch.zeros(2, dtype=torch.int32)), stream=types.SimpleNamespace(device_index=0, cuda_stream=7))
    for bad in (dict(logits=Fake(torch.zeros(2, 16, dtype=torch.float16))), dict(logits=Fake(torch.zeros(16))), dict(logits=torch.zeros(2, 16)),
                dict(logits=Fake(torch.zeros(16, 2).T)), dict(u=Fake(torch.zeros(3))), dict(u=Fake(torch.zeros(2), 0)), dict(u=Fake(torch.zeros(2, dtype=torch.float64))),
                dict(temperature=Fake(torch.zeros(3))), dict(top_k=Fake(torch.zeros(2))), dict(top_p=Fake(torch.zeros(4)[::2])),
                dict(min_p=Fake(torch.zeros(2), 0)), dict(out=Fake(torch.zeros(2)))):
        with pytest.raises(ValueError):
            sampling.sample(**{"logits": z, "u": u, **bad})
    assert calls == []


def test_numbers_as_settings(machine, monkeypatch):
    """Whatever kind of number: large top_k is not taken for another one, negative ones stay negative."""
    current, calls, _ = machine
    current[0] = 1
    got = []
    monkeypatch.setattr(sampling, "_fn", lambda *args: got.append(args[10:14]) or 0)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    z, u = Fake(torch.zeros(2, 16)), Fake(torch.zeros(2))
    for k, want in ((5, 5), (np.int64(7), 7), (2 ** 31, 2 ** 31 - 1), (2 ** 40 + 3, 2 ** 31 - 1), (-1, -1), (-2 ** 32, -1), (True, 1)):
        sampling.sample(z, u, temperature=np.float32(0.5), top_k=k, top_p=1, min_p=np.float64(0.25))
        assert got[-1] == (0.5, want, 1.0, 0.25) and [type(v) for v in got[-1]] == [float, int, float, float], got[-1]
    with pytest.raises(TypeError):
        sampling.sample(z, u, top_k=5.0)
