"""64-bit definitions of the paged-batch operators and the error bounds their tests use (plain torch, no library code)."""
from __future__ import annotations

import math
from dataclasses import dataclass, field
from typing import List, Optional

import torch

F64 = torch.float64


def half_step(dtype) -> float:
    """Largest relative error of one rounding to nearest."""
    return torch.finfo(dtype).eps / 2


@dataclass
class Batch:
    """A ragged batch over a paged pool, kept on the host; .device_args() makes what RowBatch takes."""
    n: List[int]
    kv: List[int]
    heads: int
    kv_heads: int
    dim: int
    page: int
    dtype: torch.dtype
    blocks: int = 1
    block: int = 0
    prefix_len: int = 0
    padding: int = 0                      # rows behind the last sequence
    seed: int = 0
    poison: bool = True                   # NaN in every slot that holds no position
    pool: torch.Tensor = field(init=False)

    def __post_init__(self):
        g = torch.Generator().manual_seed(1000 + self.seed)
        self.start = [0]
        for x in self.n:
            self.start.append(self.start[-1] + x)
        self.n_rows = self.start[-1] + self.padding
        per = [-(-l // self.page) for l in self.kv]
        n_prefix = -(-self.prefix_len // self.page)
        self.n_pages = sum(per) + n_prefix + 2
        perm = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.prefix_pages = perm[:n_prefix].clone()
        self.page_table = torch.full((len(self.n), max([1] + per)), 1 << 20, dtype=torch.int32)   # unused entries: no page at all
        at = n_prefix
        for i, m in enumerate(per):
            self.page_table[i, :m] = perm[at:at + m]
            at += m
        shape = (self.n_pages, self.blocks, 2, self.kv_heads, self.page, self.dim)
        self.pool = torch.full(shape, float("nan") if self.poison else 0.0).to(self.dtype)
        live = torch.randn(shape, generator=g).to(self.dtype)
        for pages, length in [(self.prefix_pages, self.prefix_len)] + [(self.page_table[i], l) for i, l in enumerate(self.kv)]:
            for p0 in range(0, length, self.page):
                m = min(self.page, length - p0)
                pg = int(pages[p0 // self.page])
                self.pool[pg, self.block, :, :, :m] = live[pg, self.block, :, :, :m]
        self.q = torch.randn(self.n_rows, self.heads, self.dim, generator=g).to(self.dtype)

    def device_args(self, dev="cuda"):
        return (torch.tensor(self.start, dtype=torch.int32, device=dev), torch.tensor(self.kv, dtype=torch.int32, device=dev),
                self.page_table.to(dev)), dict(n_rows=self.n_rows, max_rows=max([1] + self.n),
                                               prefix_pages=self.prefix_pages.to(dev), prefix_len=self.prefix_len)

    def visible(self, i: int):
        """(page, slot, own position or -1) of every position sequence i can see; positions on pages outside the pool are left out."""
        pos = [(int(self.prefix_pages[p // self.page]), p % self.page, -1) for p in range(self.prefix_len)]
        pos += [(int(self.page_table[i, p // self.page]), p % self.page, p) for p in range(self.kv[i])]
        return [x for x in pos if 0 <= x[0] < self.n_pages]


def attention(b: Batch, pool: torch.Tensor, q: torch.Tensor, scale: Optional[float] = None, dev="cpu"):
    """(out, tol): the exact result in 64 bits and the largest error the operator may make, element by element.

    With h = half a step of the storage type and u = 2^-24: the result's rounding is h |o|; the probabilities may be rounded
    to the storage type before the product with V (h each), which moves o by at most h A, A = sum p |v| / sum p; a
    score of D fp32 products is off by at most (D + 2) u s, s = scale sum |q k|, as is its difference from the maximum,
    so a probability is off by a factor of 1 + 2 (D + 4) u s at most, plus the exponential's own error, which is kept below
    h / 8; the two sums over N positions add 2 N u.  The sum of the probabilities has the same errors, hence the factor 2."""
    scale = b.dim ** -0.5 if scale is None else scale
    h, u = half_step(b.dtype), 2.0 ** -24
    out = torch.zeros(b.n_rows, b.heads, b.dim, dtype=F64, device=dev)
    tol = torch.zeros_like(out)
    G = b.heads // b.kv_heads
    pool, q = pool.to(dev), q.to(dev)
    for i, n in enumerate(b.n):
        vis = b.visible(i)
        if n == 0 or not vis:
            continue
        page, slot, own = (torch.tensor([x[j] for x in vis], device=dev) for j in range(3))
        kv = pool[page, b.block, :, :, slot].to(F64)                       # [N, 2, kv heads, dim]
        k, v = (kv[:, j].repeat_interleave(G, dim=1) for j in range(2))     # [N, heads, dim]
        x = q[b.start[i]:b.start[i] + n].to(F64)
        s = torch.einsum("rhd,nhd->hrn", x, k) * scale
        mag = torch.einsum("rhd,nhd->hrn", x.abs(), k.abs()) * scale
        last = torch.arange(n, device=dev) + (b.kv[i] - n)
        hidden = (own[None, :] >= 0) & (own[None, :] > last[:, None])      # every row sees the whole prefix
        s = s.masked_fill(hidden[None], -math.inf)
        top = s.amax(-1, keepdim=True)
        e = torch.exp(s - torch.where(top.isinf(), torch.zeros_like(top), top))
        l = e.sum(-1, keepdim=True)
        p = torch.where(l > 0, e / l, torch.zeros_like(e))
        o = torch.einsum("hrn,nhd->rhd", p, v)
        A = torch.einsum("hrn,nhd->rhd", p, v.abs())
        worst = mag.masked_fill(hidden[None], 0.0).amax(-1).T[..., None]     # [rows, heads, 1]
        N = len(vis)
        d = 2 * (b.dim + 4) * u * worst + h / 8 + 2 * N * u + 4 * u
        rows = slice(b.start[i], b.start[i] + n)
        out[rows] = o
        tol[rows] = h * o.abs() + (h + 2 * d) * A + (2 * d) * o.abs()
    return out, tol


def frequencies(rotary_dim, theta=10000.0, factor=1.0, original=0, low=1.0, high=4.0) -> List[float]:
    out = []
    for i in range(rotary_dim // 2):
        f = theta ** (-2.0 * i / rotary_dim)
        keep = 0.0
        if original:
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
        out.append(keep * f + (1 - keep) * f / factor)
    return out


def table(n_positions, rotary_dim, magnitude=1.0, **kw) -> torch.Tensor:
    ang = torch.outer(torch.arange(n_positions, dtype=F64), torch.tensor(frequencies(rotary_dim, **kw), dtype=F64))
    return torch.stack([ang.cos(), ang.sin()], dim=-1) * magnitude


def finish_heads(x: torch.Tensor, pos: torch.Tensor, freq: Optional[List[float]], interleaved: bool, gain, eps: float):
    """Norm and rotation of [rows, heads, dim] at positions pos; returns (result, sum of magnitudes behind each element)."""
    x = x.to(F64)
    if gain is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain.to(F64)
    y, mag = x.clone(), x.abs()
    if freq is not None:
        half = len(freq)
        a = torch.arange(half) * (2 if interleaved else 1)
        c = a + (1 if interleaved else half)
        ang = torch.outer(pos.to(F64), torch.tensor(freq, dtype=F64))[:, None]
        y[..., a] = x[..., a] * ang.cos() - x[..., c] * ang.sin()
        y[..., c] = x[..., c] * ang.cos() + x[..., a] * ang.sin()
        mag = x.abs()
        both = mag[..., a] + mag[..., c]
        mag[..., a], mag[..., c] = both, both
    return y, mag


def append_tolerance(ref, mag, dim, dtype):
    """One rounding to the cache's type; in fp32 the norm's sum of dim squares and its root, the gain, two products with
    rounded cos and sin and a sum: at most (dim / 2 + 12) steps of 2^-24 of the magnitudes involved."""
    return half_step(dtype) * ref.abs() + (dim / 2 + 12) * 2.0 ** -24 * (1 + half_step(dtype)) * mag + 2.0 ** -25 * (dtype == torch.float16)
