"""ctypes binding of the 4-bit paged cache (ee_kv4_* of include/ee.h): argument marshalling, and the torch buffers it works in."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from .binding import EE_BF16, EE_F32, _chk, ee_kv4_arrays, ee_kv4_config, lib

_DTYPES = {EE_BF16: torch.bfloat16, EE_F32: torch.float32}
_CODES = {torch.bfloat16: EE_BF16, torch.float32: EE_F32, "bf16": EE_BF16, "f32": EE_F32, EE_BF16: EE_BF16, EE_F32: EE_F32}

_LEAST_SCALE = 2.0 ** -149  # of fp32: less would be passed as 0, which stands for the default


_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _raw_stream(stream, index: int) -> int:
    if stream is None:
        return _current_stream(index)
    if stream.device_index != index:
        raise ValueError(f"stream of device {stream.device_index}, expected cuda:{index}")
    return stream.cuda_stream


def _used_on(stream, *tensors) -> None:
    """Memory of the tensors is not given out again before what `stream` has been told to do with them is done."""
    for t in tensors:
        t.record_stream(stream)


class Kv4Cache:
    """Owns the pool, the state (torch, device) and the ee_kv4 handle.

    Arrays of the latest plan, on the device, always at the same place: slots, positions, row_seq [max_rows], row_start
    [max_seqs + 1], served, held_next [max_seqs], n_free [1]; table [max_seqs][blocks] and free [n_blocks] are the state that
    outlasts it.

    Calls run on the cache's device, whichever is current, on torch's current stream there or on `stream`; on the latter the
    caller orders them after what wrote their inputs, and what reads their results after them."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, block_tokens: int, n_blocks: int, max_seqs: int,
                 max_positions: int, max_rows: int, dtype="bf16", device="cuda:0", stream=None):
        self.h = C.c_void_p()
        if dtype not in _CODES:
            raise ValueError(f"dtype {dtype}: bf16 or f32")
        self.cfg = cfg = ee_kv4_config(n_layers, n_heads, n_kv_heads, head_dim, _CODES[dtype], block_tokens, n_blocks, max_seqs, max_positions,
                                       max_rows)
        pb, sb = C.c_size_t(), C.c_size_t()
        _chk(lib().ee_kv4_bytes(C.byref(cfg), C.byref(pb), C.byref(sb)), "ee_kv4_bytes")
        self.device, self.dtype = torch.device(device), _DTYPES[cfg.dtype]
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        self._index = self.device.index
        self.pool = self._empty(stream, pb.value, dtype=torch.uint8)
        self.state = self._empty(stream, sb.value, dtype=torch.uint8)
        with torch.cuda.device(self._index):
            _chk(lib().ee_kv4_create(C.byref(cfg), self.pool.data_ptr(), pb.value, self.state.data_ptr(), sb.value,
                                     _raw_stream(stream, self._index), C.byref(self.h)), "ee_kv4_create")
        a = ee_kv4_arrays()
        _chk(lib().ee_kv4_get_arrays(self.h, C.byref(a)), "ee_kv4_get_arrays")

        def view(ptr: int, n: int, dt) -> torch.Tensor:
            at = ptr - self.state.data_ptr()
            return self.state[at:at + n * dt.itemsize].view(dt)

        self.table = view(a.table, max_seqs * a.table_stride, torch.int32).view(max_seqs, a.table_stride)
        self.free = view(a.free_blocks, n_blocks, torch.int32)
        self.slots = view(a.slots, max_rows, torch.int64)
        self.positions = view(a.positions, max_rows, torch.int32)
        self.row_seq = view(a.row_seq, max_rows, torch.int32)
        self.row_start = view(a.row_start, max_seqs + 1, torch.int32)
        self.served = view(a.served, max_seqs, torch.int32)
        self.held_next = view(a.held_next, max_seqs, torch.int32)
        self.n_free = view(a.n_free, 1, torch.int32)
        self.n_rows = 0
        # (calls of the loop over layers: looked up once)
        self._heads, self._kv_heads, self._head_dim = n_heads, n_kv_heads, head_dim
        L = lib()
        self._plan, self._append, self._read, self._attend = L.ee_kv4_plan, L.ee_kv4_append, L.ee_kv4_read, L.ee_kv4_attend

    def _empty(self, stream, *shape, dtype) -> torch.Tensor:
        if stream is None:
            return torch.empty(*shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(stream):
            t = torch.empty(*shape, dtype=dtype, device=self.device)
        _used_on(torch.cuda.current_stream(self.device), t)  # where the caller will want it
        return t

    def _lengths(self, t: torch.Tensor, n: int, what: str) -> int:
        if t.dtype is not torch.int32 or t.get_device() != self._index or t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{what}: int32[{n}] on {self.device}, contiguous")
        return t.data_ptr()

    def _vectors(self, t: torch.Tensor, heads: int, rows: Optional[int], what: str) -> Tuple[int, int, int]:
        if t.dtype is not self.dtype or t.get_device() != self._index or t.dim() != 3:
            raise ValueError(f"{what}: {self.dtype} [rows][heads][head_dim] on {self.device}")
        n, h, d = t.shape
        if h != heads or d != self._head_dim or (rows is not None and n != rows):
            raise ValueError(f"{what}: shape {tuple(t.shape)}, expected [{'rows' if rows is None else rows}][{heads}][{self.cfg.head_dim}]")
        sr, sh, sd = t.stride()
        if sd != 1:
            raise ValueError(f"{what}: the elements of a head must be contiguous")
        return t.data_ptr(), sr, sh

    def plan(self, held: torch.Tensor, start: torch.Tensor, end: torch.Tensor, n_rows: int, max_rows_per_seq: Optional[int] = None,
             stream=None) -> None:
        """ee_kv4_plan.  held, start, end: int32[n_seqs] on the device; max_rows_per_seq: n_rows where it is not given (the
        attention then works as for long chunks: give 1 for a plain decode step)."""
        if _current_device() != self._index:  # (the default stream's handle is 0 on every device: a launch goes to the current one)
            with torch.cuda.device(self._index):
                return self.plan(held, start, end, n_rows, max_rows_per_seq, stream)
        n = held.shape[0]
        code = self._plan(self.h, n, self._lengths(held, n, "held"), self._lengths(start, n, "start"), self._lengths(end, n, "end"), n_rows,
                          n_rows if max_rows_per_seq is None else max_rows_per_seq, _raw_stream(stream, self._index))
        if code:
            _chk(code, "ee_kv4_plan")
        if stream is not None:
            _used_on(stream, held, start, end)
        self.n_rows = n_rows

    def _slot_ptr(self, slots: torch.Tensor, rows: int) -> int:
        if slots.dtype is not torch.int64 or slots.get_device() != self._index or slots.shape != (rows,) or not slots.is_contiguous():
            raise ValueError(f"slots: int64[{rows}] on {self.device}, contiguous")
        return slots.data_ptr()

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, slots: Optional[torch.Tensor] = None, stream=None) -> None:
        """ee_kv4_append.  k, v: [rows][n_kv_heads][head_dim], any strides of rows and heads; slots: the latest plan's where not
        given."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.append(layer, k, v, slots, stream)
        rows = k.shape[0]
        kp, kr, kh = self._vectors(k, self._kv_heads, None, "k")
        vp, vr, vh = self._vectors(v, self._kv_heads, rows, "v")
        code = self._append(self.h, layer, rows, kp, kr, kh, vp, vr, vh, None if slots is None else self._slot_ptr(slots, rows),
                            _raw_stream(stream, self._index))
        if code:
            _chk(code, "ee_kv4_append")
        if stream is not None:
            _used_on(stream, k, v, *(() if slots is None else (slots,)))

    def read(self, layer: int, slots: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """ee_kv4_read -> k, v [rows][n_kv_heads][head_dim]: the values that the slots hold."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.read(layer, slots, stream)
        rows = slots.shape[0]
        p = self._slot_ptr(slots, rows)
        k = self._empty(stream, rows, self._kv_heads, self._head_dim, dtype=self.dtype)
        v = self._empty(stream, rows, self._kv_heads, self._head_dim, dtype=self.dtype)
        code = self._read(self.h, layer, rows, p, k.data_ptr(), v.data_ptr(), _raw_stream(stream, self._index))
        if code:
            _chk(code, "ee_kv4_read")
        if stream is not None:
            _used_on(stream, slots)
        return k, v

    def attend(self, layer: int, q: torch.Tensor, scale: Optional[float] = None, window: int = 0, lse: bool = False,
               out: Optional[torch.Tensor] = None, stream=None):
        """ee_kv4_attend -> [rows][n_heads][head_dim], with lse=True also log sum exp [rows][n_heads].  q: the rows of the latest
        plan, any strides of rows and heads; scale: 1 / sqrt(head_dim) where not given."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.attend(layer, q, scale, window, lse, out, stream)
        if scale is not None and not scale >= _LEAST_SCALE:
            raise ValueError("scale: positive, in fp32")
        heads, hd = self._heads, self._head_dim
        qp, qr, qh = self._vectors(q, heads, self.n_rows, "q")
        if out is None:
            out = self._empty(stream, self.n_rows, heads, hd, dtype=self.dtype)
        elif out.dtype != self.dtype or out.device != self.device or out.shape != (self.n_rows, heads, hd) or not out.is_contiguous():
            raise ValueError(f"out: {self.dtype} [{self.n_rows}][{heads}][{hd}] on {self.device}, contiguous")
        s = self._empty(stream, self.n_rows, heads, dtype=torch.float32) if lse else None
        code = self._attend(self.h, layer, qp, qr, qh, out.data_ptr(), s.data_ptr() if lse else None, scale or 0.0, window,
                            _raw_stream(stream, self._index))
        if code:
            _chk(code, "ee_kv4_attend")
        if stream is not None:
            _used_on(stream, q, out)
        return (out, s) if lse else out

    def close(self) -> None:
        if self.h:
            torch.cuda.synchronize(self.device)
            lib().ee_kv4_free(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
