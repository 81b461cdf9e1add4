"""ctypes binding of ee_sample (include/ee.h): argument marshalling only."""
from __future__ import annotations

import ctypes as C
from numbers import Real
from operator import index as index_of
from typing import Optional, Union

import torch

from .binding import EE_BF16, EE_F32, _chk, lib
from .kv4 import _current_device, _raw_stream, _used_on

_CODES = {torch.bfloat16: EE_BF16, torch.float32: EE_F32}
_fn, _sizes = None, {}


def _workspace_bytes(rows: int, vocab: int, cuts: bool) -> int:
    size = _sizes.get((rows, vocab, cuts))
    if size is None:
        s = C.c_size_t()
        query = "ee_sample_bytes" if cuts else "ee_sample_uncut_bytes"
        _chk(getattr(lib(), query)(rows, vocab, C.byref(s)), query)
        if len(_sizes) >= 4096:
            _sizes.clear()
        size = _sizes[(rows, vocab, cuts)] = s.value
    return size


def _setting(v, off, dtype, rows: int, index: int, what: str):
    """-> (address or None, number) of a setting: one per row, or one for all."""
    if v is None:
        return None, off
    if isinstance(v, Real):
        if dtype is torch.int32:  # (what has no room in it stays as large, or as wrong)
            return None, max(min(index_of(v), 2 ** 31 - 1), -1)
        return None, float(v)
    if v.dtype is not dtype or v.get_device() != index or v.shape != (rows,) or not v.is_contiguous():
        raise ValueError(f"{what}: {dtype}[{rows}] on cuda:{index}, contiguous, or a number")
    return v.data_ptr(), off


def sample(logits: torch.Tensor, u: torch.Tensor, temperature: Union[None, float, torch.Tensor] = None, top_k: Union[None, int, torch.Tensor] = None,
           top_p: Union[None, float, torch.Tensor] = None, min_p: Union[None, float, torch.Tensor] = None, scores: bool = False,
           out: Optional[torch.Tensor] = None, stream=None):
    """ee_sample -> tokens int32 [rows]; with scores=True also the tokens' log-probabilities and the confidences (the largest
    probability of each row), fp32 [rows], both under the logits as they are.

    logits: [rows][vocab], bf16 or f32, any stride of rows; u: fp32 [rows] in [0, 1); temperature, top_p, min_p: fp32 [rows], top_k: int32 [rows], or a
    number for all rows, or None (temperature 1, the others off).  Runs on the logits' device, whichever is current, on torch's current
    stream there or on `stream`; on the latter the caller orders it after what wrote its inputs, and what reads its results after it."""
    global _fn
    index = logits.get_device()
    if logits.dtype not in _CODES or logits.dim() != 2 or index < 0:
        raise ValueError(f"logits: bf16 or f32 [rows][vocab] on a GPU, not {logits.dtype} {tuple(logits.shape)} on {logits.device}")
    if _current_device() != index:  # (the default stream's handle is 0 on every device: a launch goes to the current one)
        with torch.cuda.device(index):
            return sample(logits, u, temperature, top_k, top_p, min_p, scores, out, stream)
    rows, vocab = logits.shape
    if vocab > 1 and logits.stride(1) != 1:
        raise ValueError("logits: the elements of a row must be contiguous")
    if u.dtype is not torch.float32 or u.get_device() != index or u.shape != (rows,) or not u.is_contiguous():
        raise ValueError(f"u: float32[{rows}] on cuda:{index}, contiguous")
    raw = _raw_stream(stream, index)
    tp, t = _setting(temperature, 1.0, torch.float32, rows, index, "temperature")
    kp, k = _setting(top_k, 0, torch.int32, rows, index, "top_k")
    pp, p = _setting(top_p, 1.0, torch.float32, rows, index, "top_p")
    mp, m = _setting(min_p, 0.0, torch.float32, rows, index, "min_p")

    def empty(dtype, n=rows):
        if stream is None:
            return torch.empty(n, dtype=dtype, device=logits.device)
        with torch.cuda.stream(stream):
            e = torch.empty(n, dtype=dtype, device=logits.device)
        _used_on(torch.cuda.current_stream(logits.device), e)  # where the caller will want it
        return e

    if out is None:
        out = empty(torch.int32)
    elif out.dtype is not torch.int32 or out.get_device() != index or out.shape != (rows,) or not out.is_contiguous():
        raise ValueError(f"out: int32[{rows}] on cuda:{index}, contiguous")
    lp, cf = (empty(torch.float32), empty(torch.float32)) if scores else (None, None)
    if _fn is None:
        _fn = lib().ee_sample
    # (settings that cut nothing, as numbers)
    size = _workspace_bytes(rows, vocab, not (kp is pp is mp is None and (k == 0 or k >= vocab) and p == 1.0 and m == 0.0))
    work = empty(torch.uint8, size)
    code = _fn(rows, vocab, _CODES[logits.dtype], logits.data_ptr(), logits.stride(0), u.data_ptr(), tp, kp, pp, mp, t, k, p, m, out.data_ptr(),
               lp.data_ptr() if scores else None, cf.data_ptr() if scores else None,
               work.data_ptr(), size, raw)
    if code:
        _chk(code, "ee_sample")
    if stream is not None:
        _used_on(stream, logits, u, out, *(a for a in (temperature, top_k, top_p, min_p) if a is not None and not isinstance(a, Real)))
    return (out, lp, cf) if scores else out
