"""64-bit definitions of the operators over an 8-bit paged cache and the error bounds their tests use (plain torch, no library code)."""
from __future__ import annotations

import math
from dataclasses import dataclass, field
from typing import List, Optional

import torch

from paged_reference import F64, half_step

I8, E4M3 = torch.int8, torch.float8_e4m3fn
LARGEST = {I8: 127.0, E4M3: 448.0}


def as_codes(x: torch.Tensor, dtype) -> torch.Tensor:
    """The nearest codes (e4m3 has no finite one beyond 448)."""
    return x.round().clamp(-127, 127).to(I8) if dtype == I8 else x.float().clamp(-448, 448).to(E4M3)


@dataclass
class Batch8:
    """A ragged batch over a paged pool of 8-bit codes, kept on the host."""
    n: List[int]
    kv: List[int]
    heads: int
    kv_heads: int
    dim: int
    page: int
    codes: torch.dtype
    x: torch.dtype = torch.bfloat16
    blocks: int = 1
    block: int = 0
    prefix_len: int = 0
    padding: int = 0
    seed: int = 0
    spread: float = 1.0                   # scales vary by up to 2^spread either way
    pool: torch.Tensor = field(init=False)
    scales: torch.Tensor = field(init=False)

    def __post_init__(self):
        g = torch.Generator().manual_seed(3000 + self.seed)
        self.start = [0]
        for x in self.n:
            self.start.append(self.start[-1] + x)
        self.n_rows = self.start[-1] + self.padding
        per = [-(-l // self.page) for l in self.kv]
        n_prefix = -(-self.prefix_len // self.page)
        self.n_pages = sum(per) + n_prefix + 2
        perm = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.prefix_pages = perm[:n_prefix].clone()
        self.page_table = torch.full((len(self.n), max([1] + per)), 1 << 20, dtype=torch.int32)
        at = n_prefix
        for i, m in enumerate(per):
            self.page_table[i, :m] = perm[at:at + m]
            at += m
        shape = (self.n_pages, self.blocks, 2, self.kv_heads, self.page, self.dim)
        # whatever a slot may hold that has no position: the largest code, or the code of NaN; scales of unused pages are NaN
        self.pool = torch.full(shape, 127, dtype=torch.uint8).view(self.codes)
        self.scales = torch.full(shape[:4], float("nan"))
        live = as_codes(torch.randn(shape, generator=g) * (40.0 if self.codes == I8 else 100.0), self.codes).view(torch.uint8)
        bytes_ = self.pool.view(torch.uint8)
        for pages, length in [(self.prefix_pages, self.prefix_len)] + [(self.page_table[i], l) for i, l in enumerate(self.kv)]:
            for p0 in range(0, length, self.page):
                m = min(self.page, length - p0)
                pg = int(pages[p0 // self.page])
                bytes_[pg, self.block, :, :, :m] = live[pg, self.block, :, :, :m]
                size = 2.0 ** (self.spread * (2 * torch.rand(2, self.kv_heads, generator=g) - 1))
                self.scales[pg, self.block] = size * (1 / 40.0 if self.codes == I8 else 1 / 100.0)
        self.q = torch.randn(self.n_rows, self.heads, self.dim, generator=g).to(self.x)

    def device_args(self, dev="cuda"):
        return (torch.tensor(self.start, dtype=torch.int32, device=dev), torch.tensor(self.kv, dtype=torch.int32, device=dev),
                self.page_table.to(dev)), dict(n_rows=self.n_rows, max_rows=max([1] + self.n),
                                               prefix_pages=self.prefix_pages.to(dev), prefix_len=self.prefix_len)

    def visible(self, i: int):
        pos = [(int(self.prefix_pages[p // self.page]), p % self.page, -1) for p in range(self.prefix_len)]
        pos += [(int(self.page_table[i, p // self.page]), p % self.page, p) for p in range(self.kv[i])]
        return [x for x in pos if 0 <= x[0] < self.n_pages]


def attention8(b: Batch8, pool: torch.Tensor, scales: torch.Tensor, q: torch.Tensor, scale: Optional[float] = None, dev="cpu"):
    """(out, tol): the exact result in 64 bits and the largest error the operator may make, element by element.

    With u = 2^-24, h = half a step of the result's type.  Tensor cores (16-bit q): codes and q are exact operands (q's rows are brought
    to fp16 by powers of two, which loses less than 2^-38 of a row's largest element, below the sums' own rounding); a score of D fp32
    products and its two scales is off by at most (D + 6) u s, s = scale sum |q k|, and so is its difference from the maximum; log2 of V's
    scale (at most 50) and the sum of it with a maximum of at most 256 are off by 2^-16 together; the exponential is kept within 2^-14: a
    weight w = p sv is off by a factor of 1 + d, d = 2 (D + 8) u s + 2^-15 + 2^-14, and its rounding to fp16 adds 2^-11, or 2^-32 of the
    row's largest weight.  The sums over N positions add 2 N u, and the sum of the weights has the same errors as they: factor 2.
    fp32 arithmetic (fp32 q): no rounding of the weights, values code x scale off by u, the exponential's error 4 u.
    fp16 results below 2^-14 are off by up to half a subnormal step, 2^-25."""
    scale = b.dim ** -0.5 if scale is None else scale
    tc = b.x != torch.float32
    h, u = half_step(b.x), 2.0 ** -24
    out = torch.zeros(b.n_rows, b.heads, b.dim, dtype=F64, device=dev)
    tol = torch.zeros_like(out)
    G = b.heads // b.kv_heads
    bytes_, scales, q = pool.to(dev).view(torch.uint8), scales.to(dev), q.to(dev)
    for i, n in enumerate(b.n):
        vis = b.visible(i)
        if n == 0 or not vis:
            continue
        page, slot, own = (torch.tensor([x[j] for x in vis], device=dev) for j in range(3))
        code = bytes_[page, b.block, :, :, slot].contiguous().view(pool.dtype).to(F64)          # [N, 2, kv heads, dim]
        sc = scales[page, b.block].to(F64)                                                      # [N, 2, kv heads]
        k, v = ((code[:, j] * sc[:, j, :, None]).repeat_interleave(G, dim=1) for j in range(2))  # [N, heads, dim]
        sv, cv = sc[:, 1].repeat_interleave(G, dim=1).T[:, None], code[:, 1].abs().repeat_interleave(G, dim=1)
        x = q[b.start[i]:b.start[i] + n].to(F64)
        s = torch.einsum("rhd,nhd->hrn", x, k) * scale
        mag = torch.einsum("rhd,nhd->hrn", x.abs(), k.abs()) * scale
        last = torch.arange(n, device=dev) + (b.kv[i] - n)
        hidden = ((own[None, :] >= 0) & (own[None, :] > last[:, None]))[None]
        s = s.masked_fill(hidden, -math.inf)
        top = s.amax(-1, keepdim=True)
        e = torch.exp(s - torch.where(top.isinf(), torch.zeros_like(top), top))
        l = e.sum(-1, keepdim=True)
        p = torch.where(l > 0, e / l, torch.zeros_like(e))
        o = torch.einsum("hrn,nhd->rhd", p, v)
        A = torch.einsum("hrn,nhd->rhd", p, v.abs())
        worst = mag.masked_fill(hidden, 0.0).amax(-1).T[..., None]
        N = len(vis)
        if tc:
            w = p * sv
            most = torch.einsum("hr,hrn,nhd->rhd", w.amax(-1), (~hidden).expand_as(w).to(F64), cv)
            d = 2 * (b.dim + 8) * u * worst + 2.0 ** -15 + 2.0 ** -14 + 2 * N * u
            t = h * o.abs() + (2.0 ** -11 + 2 * d) * A + 2 * d * o.abs() + 2.0 ** -32 * most
        else:
            d = 2 * (b.dim + 8) * u * worst + 2 * N * u + 8 * u
            t = h * o.abs() + 2 * d * (A + o.abs())
        rows = slice(b.start[i], b.start[i] + n)
        out[rows], tol[rows] = o, t + (2.0 ** -25 if b.x == torch.float16 else 0.0)
    return out, tol


def finish8(x, pos, table, interleaved, gain, eps):
    """Norm and rotation of [rows, heads, dim] by the table's rows pos, in 64 bits."""
    x = x.to(F64)
    if gain is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain.to(F64)
    y = x.clone()
    if table is not None:
        half = table.shape[1]
        a = torch.arange(half) * (2 if interleaved else 1)
        c = a + (1 if interleaved else half)
        t = table.to(F64)[pos][:, None]
        y[..., a] = x[..., a] * t[..., 0] - x[..., c] * t[..., 1]
        y[..., c] = x[..., c] * t[..., 0] + x[..., a] * t[..., 1]
    return y


def append8(b: Batch8, pool, scales, k, v, table=None, interleaved=False, gain=None, eps=1e-5, positions=None):
    """Pool and scales after an append of k, v, and what the tests allow for: (codes as F64 [..], scales, borderline).  A code may differ by one
    where x / scale lies within 2^-40 of the border between two (both sides work in 64 bits)."""
    dt = pool.dtype
    code, scales = pool.to(F64).clone(), scales.clone()
    width, P = b.page_table.shape[1], b.page
    near = torch.zeros(code.shape, dtype=torch.bool)
    for i, n in enumerate(b.n):
        own = torch.arange(n) + b.kv[i] - n
        rows = torch.arange(n) + b.start[i]
        keep = (own >= 0) & (own < width * P)
        own, rows = own[keep], rows[keep]
        if not len(own):
            continue
        pages = b.page_table[i].long()[own // P]
        pos = own + b.prefix_len if positions is None else positions[rows].long()
        keep = (pages >= 0) & (pages < b.n_pages)
        if table is not None:
            keep &= (pos >= 0) & (pos < table.shape[0])
        own, rows, pages, pos = own[keep], rows[keep], pages[keep], pos[keep]
        kf = finish8(k[rows], pos, table, interleaved, gain, eps)
        x = torch.stack([kf, v[rows].to(F64)], 1)                          # [rows, 2, kv heads, dim]
        for pg in pages.unique().tolist():
            mine = pages == pg
            fresh = int(own[mine].min()) // P * P >= b.kv[i] - n
            need = (x[mine].abs().amax((0, 3)) / LARGEST[dt]).float()
            need = torch.where(need < 2.0 ** -50, torch.zeros_like(need), need)
            had = torch.zeros_like(need) if fresh else scales[pg, b.block]
            new = torch.maximum(had, need)
            new = torch.where(~(need <= 2.0 ** 50) | ~(had >= 0), torch.full_like(new, math.nan), new)
            inv = torch.where(new > 0, 1.0 / new.to(F64), 0.0)
            ratio = torch.where(new > 0, had.to(F64) / new.to(F64), 0.0)
            held = torch.where(ratio[..., None, None] > 0, code[pg, b.block] * ratio[..., None, None], 0.0)
            held = torch.where((had == new)[..., None, None] & (not fresh), code[pg, b.block], as_codes(held, dt).to(F64))
            t = (x[mine] * inv[None, ..., None]).nan_to_num(0.0)
            held[:, :, own[mine] % P] = as_codes(t, dt).to(F64).permute(1, 2, 0, 3)
            code[pg, b.block] = held
            scales[pg, b.block] = new
            if dt == I8:
                near[pg, b.block][:, :, own[mine] % P] = ((t - t.floor() - 0.5).abs() < 2.0 ** -40).permute(1, 2, 0, 3)
    return code, scales, near
