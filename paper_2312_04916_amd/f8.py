"""ctypes binding of products with weights held in 8 bits (ee_f8_* of include/ee.h): argument marshalling, and the packed weight's buffer."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import EE_BF16, EE_F32, _chk, lib
from .kv4 import _current_device, _raw_stream, _used_on

_CODES = {torch.bfloat16: EE_BF16, torch.float32: EE_F32}


def _rows(t: torch.Tensor, index: int, rows: Optional[int], cols: int, what: str):
    """-> (address, row stride) of rows that a call reads or writes."""
    if t.dtype not in _CODES or t.get_device() != index or t.dim() != 2 or t.shape[1] != cols or (rows is not None and t.shape[0] != rows):
        raise ValueError(f"{what}: bf16 or f32 [{'rows' if rows is None else rows}][{cols}] on cuda:{index}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    return t.data_ptr(), t.stride(0)


class F8Weight:
    """A weight [n][k] packed into 8 bits an element, on its device; with `up`, a gate and an up weight side by side.

    Calls run on the weight's device, whichever is current, on torch's current stream there or on `stream`; on the latter the
    caller orders them after what wrote their inputs, and what reads their results after them."""

    def __init__(self, w: torch.Tensor, up: Optional[torch.Tensor] = None, stream=None):
        if w.dim() != 2 or not w.is_cuda:
            raise ValueError("w: [n][k] on a GPU")
        self.n, self.k, self.pair = w.shape[0], w.shape[1], up is not None
        self.device, self._index = w.device, w.get_device()
        wp, wr = _rows(w, self._index, None, self.k, "w")
        upp, upr = (None, 0) if up is None else _rows(up, self._index, self.n, self.k, "up")
        if up is not None and up.dtype != w.dtype:
            raise ValueError(f"up: {w.dtype}, as w")
        size = C.c_size_t()
        _chk(lib().ee_f8_bytes(self.n, self.k, self.pair, C.byref(size)), "ee_f8_bytes")
        self.packed = self._empty(stream, size.value, dtype=torch.uint8)
        with torch.cuda.device(self._index):
            _chk(lib().ee_f8_pack(self.n, self.k, self.pair, _CODES[w.dtype], wp, wr, upp, upr, self.packed.data_ptr(), size.value,
                                  _raw_stream(stream, self._index)), "ee_f8_pack")
        if stream is not None:
            _used_on(stream, w, *(() if up is None else (up,)))
        # (calls of the loop over layers: looked up once)
        self._matmul, self._address, self._work = lib().ee_f8_matmul, self.packed.data_ptr(), {}

    def _empty(self, stream, *shape, dtype) -> torch.Tensor:
        if stream is None:
            return torch.empty(*shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(stream):
            t = torch.empty(*shape, dtype=dtype, device=self.device)
        _used_on(torch.cuda.current_stream(self.device), t)  # where the caller will want it
        return t

    def _workspace_bytes(self, m: int, code: int) -> int:
        size = self._work.get((m, code))
        if size is None:
            s = C.c_size_t()
            _chk(lib().ee_f8_matmul_bytes(m, self.n, self.k, self.pair, code, C.byref(s)), "ee_f8_matmul_bytes")
            if len(self._work) >= 4096:
                self._work.clear()
            size = self._work[(m, code)] = s.value
        return size

    def matmul(self, x: torch.Tensor, add: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
        """ee_f8_matmul -> [m][n]: x W^T, or silu(x Wgate^T) * (x Wup^T) of a pair.  x: [m][k], bf16 or f32, any stride of rows;
        dtype: of the result (out's, else x's); add: [m][n] of that dtype, added before the rounding; out: where the result goes
        (add itself, or apart from it)."""
        if _current_device() != self._index:  # (the default stream's handle is 0 on every device: a launch goes to the current one)
            with torch.cuda.device(self._index):
                return self.matmul(x, add, dtype, out, stream)
        raw = _raw_stream(stream, self._index)
        xp, xr = _rows(x, self._index, None, self.k, "x")
        m = x.shape[0]
        if out is None:
            dtype = x.dtype if dtype is None else dtype
            if dtype not in _CODES:
                raise ValueError(f"dtype {dtype}: bf16 or f32")
            out = self._empty(stream, m, self.n, dtype=dtype)
            op, orow = out.data_ptr(), self.n
        else:
            if dtype is not None and out.dtype != dtype:
                raise ValueError(f"out: {out.dtype}, dtype {dtype}")
            op, orow = _rows(out, self._index, m, self.n, "out")
        ap, ar = None, 0
        if add is not None:
            if add.dtype != out.dtype:
                raise ValueError(f"add: {out.dtype}, as the result")
            ap, ar = _rows(add, self._index, m, self.n, "add")
        code = _CODES[out.dtype]
        size = self._workspace_bytes(m, code)
        work = self._empty(stream, size, dtype=torch.uint8) if size else None
        rc = self._matmul(m, self.n, self.k, self.pair, self._address, _CODES[x.dtype], xp, xr, code, op, orow, ap, ar,
                          work.data_ptr() if size else None, size, raw)
        if rc:
            _chk(rc, "ee_f8_matmul")
        if stream is not None:
            _used_on(stream, self.packed, x, out, *(() if add is None else (add,)))
        return out

    def values(self, dtype: torch.dtype = torch.float32, stream=None):
        """ee_f8_unpack -> the values that the weight holds, [n][k]; of a pair both."""
        if dtype not in _CODES:
            raise ValueError(f"dtype {dtype}: bf16 or f32")
        got = [self._empty(stream, self.n, self.k, dtype=dtype) for _ in range(1 + self.pair)]
        with torch.cuda.device(self._index):
            for up, w in enumerate(got):
                _chk(lib().ee_f8_unpack(self.n, self.k, self.pair, up, self._address, _CODES[dtype], w.data_ptr(), _raw_stream(stream, self._index)),
                     "ee_f8_unpack")
        if stream is not None:
            _used_on(stream, self.packed)
        return tuple(got) if self.pair else got[0]
