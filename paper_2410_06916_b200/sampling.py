"""A token per row of logits: the torch side of swift_sample_rows (include/swift.h says what it computes).  As in paged.py, torch only
provides memory and streams; the call enqueues one hand-written kernel and returns without waiting."""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Tuple, Union

import torch

from .binding import lib
from .paged import _TYPES, _check, _cuda_tensor, _gradient, _number, _on


class _Sample(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("logits", C.c_void_p), ("row_stride", C.c_int64),
                ("uniforms", C.c_void_p), ("temperature", C.c_void_p), ("temperature_all", C.c_float), ("top_k", C.c_void_p),
                ("top_k_all", C.c_int32), ("top_p", C.c_void_p), ("top_p_all", C.c_float), ("min_p", C.c_void_p), ("min_p_all", C.c_float),
                ("tokens", C.c_void_p), ("probs", C.c_void_p)]


def _per_row(name: str, t: torch.Tensor, rows: int, device: torch.device, dtype: torch.dtype) -> int:
    _cuda_like(name, t, device)
    if t.requires_grad:
        _gradient(name)
    if t.dtype != dtype or tuple(t.shape) != (rows,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} [{rows}]")
    return t.data_ptr()


def _cuda_like(name: str, t: torch.Tensor, device: torch.device) -> None:
    _cuda_tensor(name, t)
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the logits on {device}")


def sample_rows(logits: torch.Tensor, uniforms: torch.Tensor, temperature: Union[float, torch.Tensor] = 1.0,
                top_k: Union[int, torch.Tensor] = 0, top_p: Union[float, torch.Tensor] = 1.0, min_p: Union[float, torch.Tensor] = 0.0,
                tokens: Optional[torch.Tensor] = None, probs: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(tokens int32 [rows], probs fp32 [rows]): a token drawn per row of logits [rows, vocab] (fp32, bf16 or fp16, dims contiguous) with
    the row's number of `uniforms`, fp32 [rows] in [0, 1), and its probability among what the filters keep.

    temperature  0 takes the largest logit, the lowest id among equals
    top_k        keeps that many of the largest logits (0 or less: all), ties to the lowest ids
    top_p        keeps of those the fewest, largest first, that hold this share of their probability (1: all)
    min_p        keeps of those the ones at least this probable, relative to the most probable (0: all)
    Each is a number for all rows, or a tensor [rows] on the device (int32 for top_k, else fp32), read when the work runs: a
    captured call follows its new values.

    A row without an answer gets token -1 and probability 0: logits with NaN or +infinity, or nothing but -infinity, a uniform outside
    [0, 1), a temperature that is negative or not finite, min_p above 1, NaN in any of them.  The same row gives the same token whatever other rows
    there are."""
    _cuda_tensor("logits", logits)
    if logits.dim() != 2 or logits.dtype not in _TYPES:
        raise ValueError("logits must be [rows, vocab] in fp32, bf16 or fp16")
    if logits.requires_grad:
        _gradient("logits")
    rows, vocab = logits.shape
    if vocab > 1 and logits.stride(1) != 1:
        raise ValueError("a row's logits must be contiguous")
    device = logits.device
    desc = _Sample(n_rows=_number("rows", rows), vocab=_number("vocab", vocab), dtype=_TYPES[logits.dtype], logits=logits.data_ptr(),
                   row_stride=logits.stride(0) if rows > 1 else vocab, uniforms=_per_row("uniforms", uniforms, rows, device, torch.float32))
    used = [logits, uniforms]
    for name, value in (("temperature", temperature), ("top_p", top_p), ("min_p", min_p), ("top_k", top_k)):
        if isinstance(value, torch.Tensor):
            setattr(desc, name, _per_row(name, value, rows, device, torch.int32 if name == "top_k" else torch.float32))
            used.append(value)
            continue
        if name == "top_k":
            _number(name, value)
        elif not (0.0 <= value < math.inf) or (name == "min_p" and value > 1.0):
            raise ValueError(f"{name} {value}")
        setattr(desc, name + "_all", value)
    for name, t, dtype in (("tokens", tokens, torch.int32), ("probs", probs, torch.float32)):
        if t is not None:
            _per_row(name, t, rows, device, dtype)
    return _on(device, stream, (*used, tokens, probs), _sample, desc, tokens, probs, device)


def _sample(s: int, desc: _Sample, tokens: Optional[torch.Tensor], probs: Optional[torch.Tensor], device: torch.device):
    if tokens is None:
        tokens = torch.empty(desc.n_rows, dtype=torch.int32, device=device)
    if probs is None:
        probs = torch.empty(desc.n_rows, dtype=torch.float32, device=device)
    desc.tokens, desc.probs = tokens.data_ptr(), probs.data_ptr()
    _check(lib().swift_sample_rows(C.byref(desc), s))
    return tokens, probs
