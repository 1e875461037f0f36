"""Batches of sequences over one paged K,V cache: the torch side of swift_rope_table, swift_kv_append,
swift_prompt_attention and swift_prefix_attention (include/swift.h says what each computes).  As in binding.py, torch only
provides memory and streams; every call enqueues hand-written kernels and returns without waiting.

A program that runs several sequences keeps one PagedKV for all layers, makes a RowBatch per step (or keeps one whose
device tensors it rewrites), and calls per layer:

    q = batch.append(block, q, k, v, rope=table)      # norm + rotation of q and k, K and V into the pages
    o = batch.prompt_attention(block, q)              # whole prompts, or chunks of them
    o = batch.prefix_attention(block, q)              # a few rows per sequence behind a shared prefix
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import SwiftError, _DevBuf, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class _Kv(C.Structure):
    _fields_ = [("pool", C.c_void_p)] + [(n, C.c_int32) for n in ("dtype", "n_pages", "n_blocks", "n_kv_heads", "page_size", "head_dim")]


class _Batch(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_rows", C.c_int32), ("row_start", C.c_void_p), ("kv_len", C.c_void_p),
                ("page_table", C.c_void_p), ("table_stride", C.c_int32), ("prefix_pages", C.c_void_p), ("prefix_len", C.c_int32)]


class _Rows(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class _RopeDesc(C.Structure):
    _fields_ = [("n_positions", C.c_int32), ("rotary_dim", C.c_int32), ("theta", C.c_double), ("factor", C.c_double),
                ("original_positions", C.c_int32), ("low_turns", C.c_double), ("high_turns", C.c_double), ("magnitude", C.c_double)]


class _Append(C.Structure):
    _fields_ = [("block", C.c_int32), ("n_heads", C.c_int32), ("x_dtype", C.c_int32), ("q", _Rows), ("k", _Rows), ("v", _Rows),
                ("q_gain", C.c_void_p), ("k_gain", C.c_void_p), ("eps", C.c_float), ("rope", C.c_void_p),
                ("rope_positions", C.c_int32), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("positions", C.c_void_p),
                ("q_out", C.c_void_p)]


class _Attention(C.Structure):
    _fields_ = [("block", C.c_int32), ("n_heads", C.c_int32), ("q", _Rows), ("scale", C.c_float), ("out", C.c_void_p)]


def _check(status: int) -> None:
    if status != 0:
        raise SwiftError(status, lib().swift_batch_error().decode())


def _raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)     # the same handle without a Stream object


class _Target:
    """Makes `device` current, and `stream` if one is given: outputs and workspaces made inside then belong to that stream."""

    __slots__ = ("guards",)

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream]):
        if stream is not None and stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
        self.guards = [torch.cuda.device(device)] + ([torch.cuda.stream(stream)] if stream is not None else [])

    def __enter__(self) -> None:
        for g in self.guards:
            g.__enter__()

    def __exit__(self, *exc) -> None:
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _on(device: torch.device, stream: Optional[torch.cuda.Stream], used, call, *args):
    """call(raw stream, *args) with `device` current, on `stream` or else the device's current stream.  used: the caller's tensors
    the call's work touches (or None); those lent to another stream are marked, so that the allocator does not hand out the memory
    of one that is freed while that stream still works on it."""
    if stream is None and torch.cuda.current_device() == device.index:
        return call(_raw_stream(device.index), *args)
    with _Target(device, stream):
        result = call(_raw_stream(device.index), *args)
    if stream is not None:
        for t in used:
            if t is not None:
                t.record_stream(stream)
    return result


def _cuda_tensor(name: str, t: torch.Tensor, device: Optional[torch.device] = None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the cache on {device}")
    return t


def _number(name: str, value: int) -> int:
    """An integer that fits the C structures' 32 bits (ctypes would cut it to them)."""
    if not -(1 << 31) <= value < 1 << 31:
        raise ValueError(f"{name} {value} does not fit 32 bits")
    return value


def _gradient(name: str) -> None:
    """For a tensor that requires a gradient: the calls have no backward pass, and a result that silently drops it is wrong."""
    if torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which these calls do not have: detach it, or call under torch.no_grad()")


def _int32(name: str, t: torch.Tensor, device: torch.device) -> torch.Tensor:
    _cuda_tensor(name, t, device)
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous int32")
    return t


def rope_table(n_positions: int, rotary_dim: int, theta: float = 10000.0, factor: float = 1.0, original_positions: int = 0,
               low_turns: float = 1.0, high_turns: float = 4.0, magnitude: float = 1.0, device="cuda",
               out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """fp32 [n_positions, rotary_dim / 2, 2]: (cos, sin) of every position and pair.  factor > 1 stretches the positions: all
    alike (original_positions 0), or by parts with low_turns / high_turns as the ramp (LLaMA 3: 1 and 4; YaRN: 1 and 32,
    with magnitude = 0.1 ln(factor) + 1).  The ramp runs over the turns, as the paper defines it; common
    implementations let it run over the pair's index between the same two ends, and checkpoints made with those need that table."""
    for name, value in (("n_positions", n_positions), ("rotary_dim", rotary_dim), ("original_positions", original_positions)):
        _number(name, value)
    device = torch.device(device) if out is None else _cuda_tensor("out", out).device
    if device.type != "cuda":
        raise ValueError("rope_table needs a CUDA device")
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    if out is not None and out.requires_grad:
        _gradient("out")
    if out is not None and (out.dtype != torch.float32 or not out.is_contiguous() or tuple(out.shape) != (n_positions, rotary_dim // 2, 2)):
        raise ValueError("out must be contiguous float32 [n_positions, rotary_dim / 2, 2]")
    desc = _RopeDesc(n_positions, rotary_dim, theta, factor, original_positions, low_turns, high_turns, magnitude)
    if n_positions < 0 or rotary_dim < 2:
        raise ValueError("n_positions >= 0 and rotary_dim >= 2")
    return _on(device, stream, (out,), _rope_table, desc, device, out)


def _rope_table(s: int, desc: _RopeDesc, device: torch.device, out: Optional[torch.Tensor]) -> torch.Tensor:
    if out is None:
        out = torch.empty(desc.n_positions, desc.rotary_dim // 2, 2, dtype=torch.float32, device=device)
    if desc.n_positions > 0:
        _check(lib().swift_rope_table(C.byref(desc), out.data_ptr(), s))
    return out


class PagedKV:
    """One K,V pool for all layers: a contiguous CUDA tensor [n_pages, n_blocks, 2, n_kv_heads, page_size, head_dim] the
    caller made (fp32, bf16 or fp16); [.., 0, ..] is K, [.., 1, ..] is V."""

    def __init__(self, pool: torch.Tensor):
        _cuda_tensor("pool", pool)
        if pool.requires_grad:
            _gradient("pool")
        if pool.dim() != 6 or pool.shape[2] != 2 or not pool.is_contiguous() or pool.dtype not in _TYPES:
            raise ValueError("pool must be contiguous [n_pages, n_blocks, 2, n_kv_heads, page_size, head_dim] in fp32, bf16 or fp16")
        self.pool, self.device, self.dtype = pool, pool.device, pool.dtype
        self.n_pages, self.n_blocks, _, self.n_kv_heads, self.page_size, self.head_dim = pool.shape
        self._c = _Kv(pool.data_ptr(), _TYPES[pool.dtype], self.n_pages, self.n_blocks, self.n_kv_heads, self.page_size, self.head_dim)


class RowBatch:
    """Rows of several sequences over a PagedKV.

    row_start  int32 [n_seqs + 1]: sequence i holds rows row_start[i] .. row_start[i + 1] - 1 of the packed tensors
    kv_len     int32 [n_seqs]: cached positions of each sequence, its rows of this batch included
    page_table int32 [n_seqs, stride]: pages of each sequence's own positions
    n_rows     rows of the packed tensors (rows from row_start[-1] on are padding)
    max_rows   upper bound of the rows of one sequence; prefix_attention leaves out rows beyond it, and chooses its kernels by
               it.  The default, n_rows, is right for any batch but slow for many sequences of few rows: give the bound
               (64 one-token continuations of 8192 positions, 64 heads on 8: 59 us with max_rows 1, 102 without)
    prefix_pages, prefix_len: a prefix that all sequences continue (its pages, its length in positions)

    The tensors are read on the device when a call's work runs; they may be rewritten between calls, and between replays
    of a captured graph.  Calls work on the device's current stream, or on `stream`, which the caller has made wait for what its
    tensors still wait for; tensors lent to it may be freed at any time.

    prefix_attention divides the SMs between the prefix and the sequences' own parts before it knows their lengths: it takes
    them for 0.6 of the page table's width.  A table much wider than its sequences (the same 64 continuations with about 750 own
    positions, in a table of 4096) costs up to twice the time; one cut to the columns in use does not.
    """

    def __init__(self, kv: PagedKV, row_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor, n_rows: int,
                 max_rows: Optional[int] = None, prefix_pages: Optional[torch.Tensor] = None, prefix_len: int = 0):
        dev = kv.device
        _int32("row_start", row_start, dev)
        _int32("kv_len", kv_len, dev)
        _int32("page_table", page_table, dev)
        if row_start.dim() != 1 or kv_len.dim() != 1 or page_table.dim() != 2:
            raise ValueError("row_start [n_seqs + 1], kv_len [n_seqs], page_table [n_seqs, stride]")
        n_seqs = kv_len.shape[0]
        if row_start.shape[0] != n_seqs + 1 or page_table.shape[0] != n_seqs or page_table.shape[1] < 1:
            raise ValueError("row_start [n_seqs + 1], kv_len [n_seqs], page_table [n_seqs, stride]")
        if n_rows < 0 or prefix_len < 0 or (max_rows is not None and max_rows < 1):
            raise ValueError("n_rows and prefix_len must not be negative, max_rows at least 1")
        _number("n_rows", n_rows), _number("prefix_len", prefix_len)
        if prefix_len > 0:
            if prefix_pages is None or _int32("prefix_pages", prefix_pages, dev).numel() * kv.page_size < prefix_len:
                raise ValueError("prefix_pages must hold prefix_len positions")
        self.kv, self.n_seqs, self.n_rows = kv, n_seqs, n_rows
        self.max_rows = max(1, n_rows if max_rows is None else min(max_rows, n_rows))
        self._keep = (row_start, kv_len, page_table, prefix_pages)
        self._tensors = (kv.pool, *self._keep)
        self._c = _Batch(n_seqs, n_rows, row_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), page_table.shape[1],
                         prefix_pages.data_ptr() if prefix_len > 0 else None, prefix_len)
        self._kv_p, self._c_p = C.byref(kv._c), C.byref(self._c)
        self._lib, self._types, self._x_types, self._scale = lib(), (kv.dtype,), (kv.dtype, torch.float32), kv.head_dim ** -0.5
        self._ws_bytes = {}

    # ------------------------------------------------------------------ checks shared by the calls
    def _rows(self, name: str, t: torch.Tensor, heads: Optional[int], dtypes) -> _Rows:
        kv = self.kv
        if not isinstance(t, torch.Tensor) or t.device != kv.device:
            _cuda_tensor(name, t, kv.device)
        shape = t.shape
        if len(shape) != 3 or shape[0] != self.n_rows or shape[2] != kv.head_dim or (heads is not None and shape[1] != heads):
            raise ValueError(f"{name} must be [{self.n_rows}, {heads if heads is not None else 'heads'}, {kv.head_dim}], got {tuple(shape)}")
        if t.requires_grad:
            _gradient(name)
        if t.dtype not in dtypes:
            raise TypeError(f"{name} must be one of {dtypes}, got {t.dtype}")
        row, head, dim = t.stride()
        if dim != 1:
            raise ValueError(f"the dims of {name} must be contiguous")
        # a stride over a single row or head means nothing
        return _Rows(t.data_ptr(), row if shape[0] > 1 else shape[1] * shape[2], head if shape[1] > 1 else shape[2])

    def _gain(self, name: str, g: torch.Tensor) -> int:
        _cuda_tensor(name, g, self.kv.device)
        if g.requires_grad:
            _gradient(name)
        if g.dtype != torch.float32 or g.shape != (self.kv.head_dim,) or not g.is_contiguous():
            raise ValueError(f"{name} must be contiguous float32 [{self.kv.head_dim}]")
        return g.data_ptr()

    def _out(self, out: Optional[torch.Tensor], heads: int) -> torch.Tensor:
        kv = self.kv
        if out is None:
            return torch.empty(self.n_rows, heads, kv.head_dim, dtype=kv.dtype, device=kv.device)
        if not isinstance(out, torch.Tensor) or out.device != kv.device:
            _cuda_tensor("out", out, kv.device)
        if out.requires_grad:
            _gradient("out")
        if out.shape != (self.n_rows, heads, kv.head_dim) or out.dtype != kv.dtype or not out.is_contiguous():
            raise ValueError(f"out must be contiguous {(self.n_rows, heads, kv.head_dim)} of {kv.dtype}")
        return out

    # ------------------------------------------------------------------ the calls
    def append(self, block: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rope: Optional[torch.Tensor] = None,
               interleaved: bool = False, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None,
               eps: float = 1e-5, positions: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Norm (where a gain fp32 [head_dim] is given) and rotation (where a rope_table is given) of q and k, K and V into the
        cache's block; returns the finished q [n_rows, heads, head_dim] in the cache's type.  q, k, v: [n_rows, heads, head_dim]
        views (slices of a fused projection), fp32 or the cache's type.  Rows left out (padding, pages or positions out of
        range) keep what `out` held.  positions: int32 [n_rows], instead of prefix_len + own position."""
        kv = self.kv
        heads = kv.n_kv_heads
        rows = (self._rows("q", q, None, self._x_types), self._rows("k", k, heads, self._x_types), self._rows("v", v, heads, self._x_types))
        if q.dtype != k.dtype or q.dtype != v.dtype:
            raise TypeError("q, k and v must have one type")
        q_gain_p = None if q_gain is None else self._gain("q_gain", q_gain)
        k_gain_p = None if k_gain is None else self._gain("k_gain", k_gain)
        rope_p, rope_rows, pairs = None, 0, 0
        if rope is not None:
            _cuda_tensor("rope", rope, kv.device)
            if rope.requires_grad:
                _gradient("rope")
            shape = rope.shape
            if rope.dtype != torch.float32 or len(shape) != 3 or shape[2] != 2 or not rope.is_contiguous() or 2 * shape[1] > kv.head_dim:
                raise ValueError("rope must be a rope_table of at most head_dim dims")
            rope_p, rope_rows, pairs = rope.data_ptr(), shape[0], shape[1]
        positions_p = None
        if positions is not None:
            if tuple(_int32("positions", positions, kv.device).shape) != (self.n_rows,):
                raise ValueError(f"positions must be [{self.n_rows}]")
            positions_p = positions.data_ptr()
        a = _Append(_number("block", block), q.shape[1], _TYPES[q.dtype], *rows, q_gain_p, k_gain_p, eps, rope_p, rope_rows, 2 * pairs, 1 if interleaved else 0, positions_p, None)
        return _on(kv.device, stream, () if stream is None else (q, k, v, rope, q_gain, k_gain, positions, out, *self._tensors), self._append, a, out)

    def _append(self, s: int, a: _Append, out: Optional[torch.Tensor]) -> torch.Tensor:
        out = self._out(out, a.n_heads)
        a.q_out = out.data_ptr()
        _check(self._lib.swift_kv_append(self._kv_p, self._c_p, C.byref(a), s))
        return out

    def _attention(self, block: int, q: torch.Tensor, scale: Optional[float]) -> _Attention:
        rows = self._rows("q", q, None, self._types)
        return _Attention(_number("block", block), q.shape[1], rows, self._scale if scale is None else scale, None)

    def prompt_attention(self, block: int, q: torch.Tensor, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Causal attention of every row over the prefix and its sequence's own positions up to its own; [n_rows, heads,
        head_dim] in the cache's type.  scale defaults to head_dim ** -0.5.  Padding rows keep what `out` held."""
        return _on(self.kv.device, stream, () if stream is None else (q, out, *self._tensors), self._prompt, self._attention(block, q, scale), out)

    def _prompt(self, s: int, a: _Attention, out: Optional[torch.Tensor]) -> torch.Tensor:
        out = self._out(out, a.n_heads)
        a.out = out.data_ptr()
        _check(self._lib.swift_prompt_attention(self._kv_p, self._c_p, C.byref(a), s))
        return out

    def prefix_attention(self, block: int, q: torch.Tensor, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The same function for few rows per sequence: what all rows share of the prefix is computed once for all of them.
        Rows of a sequence beyond max_rows are left out."""
        return _on(self.kv.device, stream, () if stream is None else (q, out, *self._tensors), self._prefix, self._attention(block, q, scale), out)

    def _prefix(self, s: int, a: _Attention, out: Optional[torch.Tensor]) -> torch.Tensor:
        need = self._ws_bytes.get(a.n_heads)
        if need is None:
            need = self._lib.swift_prefix_workspace_bytes(self._kv_p, self._c_p, a.n_heads, self.max_rows)
            if need == 0:
                raise SwiftError(1, self._lib.swift_batch_error().decode())
            self._ws_bytes[a.n_heads] = need
        out = self._out(out, a.n_heads)
        a.out = out.data_ptr()
        ws = torch.empty(need, dtype=torch.uint8, device=self.kv.device)     # of this call alone; the allocator aligns to 512
        _check(self._lib.swift_prefix_attention(self._kv_p, self._c_p, C.byref(a), self.max_rows, _DevBuf(ws.data_ptr(), need), s))
        return out


def batch_sync(device="cuda", stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises SwiftError if a bounded device-side wait of an attention call ran out (ETIMEOUT)."""
    device = stream.device if stream is not None else torch.device(device)
    if device.type != "cuda":
        raise ValueError("batch_sync needs a CUDA device")
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    _on(device, stream, (), lambda s: _check(lib().swift_batch_sync(s)))
