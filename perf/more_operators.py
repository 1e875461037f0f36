"""Operators of a batch whose K,V cache is held in 8 bits, and of the token drawn at its end: what is measured, and on what.

Three operators, as a serving program chains them:
  append8   per-head norm of q and k, rotation, and K,V into the pages of an 8-bit cache, in one pass
  attend8   attention over that cache: whole prompts or chunks of them, or a few rows per sequence behind a shared prefix
  sample    a token per row from its logits: temperature, top-k, top-p and min-p, from given random numbers

The cache is one pool [page][block][K or V][kv head][slot][dim] of int8 or float8 (e4m3) codes for all layers; a page's K (or V)
of one kv head shares one scale, [page][block][K or V][kv head]: value = code x scale.
`own = False` computes them from elementary torch operations; `own = True` calls the library.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"i8": 127.0, "e4m3": 448.0}


# ----------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step of 16 sequences of the 13B shape: a token each into pages that are partly full; latency counts
        {"name": "append8 decode 13b", "op": "append8", "codes": "i8", "x": "bf16", "heads": 40, "kv_heads": 40, "dim": 128,
         "page": 16, "seqs": 16, "rows": 16, "shortest": 1, "cached": 1000, "prefix": 0, "lens_seed": 1, "rotary_dim": 128,
         "interleaved": False, "norm": False, "blocks": 2},
        # the prompts of a batch of the 70B shape with normed queries and keys, out of the fused projection
        {"name": "append8 prompts 70b", "op": "append8", "codes": "i8", "x": "bf16", "heads": 64, "kv_heads": 8, "dim": 128,
         "page": 64, "seqs": 7, "rows": 8192, "shortest": 100, "cached": 0, "prefix": 0, "lens_seed": 2, "rotary_dim": 128,
         "interleaved": False, "norm": True, "blocks": 2},
        # neighbouring pairs over half of a small head, fp32 activations into an e4m3 cache, continuing cached prompts
        {"name": "append8 pairs e4m3", "op": "append8", "codes": "e4m3", "x": "f32", "heads": 24, "kv_heads": 6, "dim": 64,
         "page": 32, "seqs": 5, "rows": 3001, "shortest": 0, "cached": 700, "prefix": 333, "lens_seed": 3, "rotary_dim": 32,
         "interleaved": True, "norm": True, "blocks": 1},
        # two sequences, a token each, heads of 64: the smallest decoding step
        {"name": "decode8 smallest", "op": "attend8", "form": "prefix", "codes": "i8", "x": "bf16", "heads": 4, "kv_heads": 4,
         "dim": 64, "page": 16, "seqs": 2, "rows": 2, "shortest": 1, "cached": 60, "prefix": 100, "lens_seed": 1, "blocks": 1},
        # a decoding step of 64 long conversations of the 70B shape
        {"name": "decode8 64 of 70b", "op": "attend8", "form": "prefix", "codes": "i8", "x": "bf16", "heads": 64, "kv_heads": 8,
         "dim": 128, "page": 64, "seqs": 64, "rows": 64, "shortest": 1, "cached": 8000, "prefix": 0, "lens_seed": 2, "blocks": 1},
        # one token behind one very long document, grouped heads
        {"name": "decode8 131k", "op": "attend8", "form": "prefix", "codes": "e4m3", "x": "bf16", "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 128, "seqs": 1, "rows": 1, "shortest": 1, "cached": 131001, "prefix": 0, "lens_seed": 1, "blocks": 1},
        # verification of 8 drafts on each of 12 sequences of the 34B shape, ragged, a short shared system prompt
        {"name": "decode8 verify 34b", "op": "attend8", "form": "prefix", "codes": "e4m3", "x": "f16", "heads": 56, "kv_heads": 8,
         "dim": 128, "page": 32, "seqs": 12, "rows": 108, "shortest": 9, "cached": 2500, "prefix": 301, "lens_seed": 5, "blocks": 1},
        # ragged prompts of the 34B shape (seven query heads on a KV head), some continuing what is cached
        {"name": "prompt8 ragged 34b", "op": "attend8", "form": "prompt", "codes": "e4m3", "x": "f16", "heads": 56, "kv_heads": 8,
         "dim": 128, "page": 16, "seqs": 9, "rows": 5003, "shortest": 1, "cached": 600, "prefix": 0, "lens_seed": 4, "blocks": 2},
        # the last 2048 tokens of a prompt of 8192 at the 70B shape, the rest in the cache already
        {"name": "prompt8 chunk 70b", "op": "attend8", "form": "prompt", "codes": "i8", "x": "bf16", "heads": 64, "kv_heads": 8,
         "dim": 128, "page": 64, "seqs": 1, "rows": 2048, "shortest": 2048, "cached": 6144, "prefix": 0, "lens_seed": 1, "blocks": 1},
        # one row of the 7B and 13B shapes' vocabulary: batch-1 decoding, every filter on; latency counts
        {"name": "sample 1 of 32000", "op": "sample", "dtype": "f32", "rows": 1, "vocab": 32000, "k": 50, "p": 0.9, "min_p": 0.02,
         "temperature": 0.8, "mixed": False, "spread": 2.5},
        # a decoding batch with a large vocabulary, nucleus sampling out of bf16 logits
        {"name": "sample 64 of 128000 bf16", "op": "sample", "dtype": "bf16", "rows": 64, "vocab": 128000, "k": 0, "p": 0.95,
         "min_p": 0.0, "temperature": 0.7, "mixed": False, "spread": 2.5},
        # the largest batch, every row with settings of its own: greedy, plain, top-k, top-p, min-p and all of them
        {"name": "sample 256 mixed", "op": "sample", "dtype": "f32", "rows": 256, "vocab": 128000, "k": 200, "p": 0.9, "min_p": 0.01,
         "temperature": 1.0, "mixed": True, "spread": 3.0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append8", "append8", "decode", "decode", "decode", "prompt", "prompt", "sample", "sample", "sample"])
    if op == "sample":
        rows, vocab = _log(rng, 1, 256), _log(rng, 1000, 128000)
        return {"op": op, "dtype": rng.choice(["f32", "f32", "bf16", "f16"]), "rows": rows, "vocab": vocab,
                "k": rng.choice([0, 0, 1, 20, 50, 1000, vocab // 3]), "p": rng.choice([1.0, 0.5, 0.9, 0.95, 0.999]),
                "min_p": rng.choice([0.0, 0.0, 0.05, 0.2]), "temperature": rng.choice([0.3, 0.7, 1.0, 1.5]),
                "mixed": rng.random() < 0.3, "spread": rng.choice([0.5, 2.0, 3.0, 5.0])}
    heads, kv_heads = rng.choice([(32, 32), (40, 40), (64, 8), (56, 8), (32, 8), (16, 2), (4, 4), (12, 1), (8, 4), (9, 3)])
    c = {"codes": rng.choice(["i8", "i8", "e4m3"]), "heads": heads, "kv_heads": kv_heads, "page": rng.choice([8, 16, 32, 64, 128]),
         "lens_seed": rng.randrange(1 << 20), "blocks": rng.choice([1, 2])}
    if op == "append8":
        c["op"] = op
        c["dim"] = rng.choice([16, 64, 80, 96, 128, 256])
        c["rotary_dim"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2])
        c["x"] = rng.choice(["bf16", "f16", "f32"])
        c["interleaved"], c["norm"] = rng.random() < 0.4, rng.random() < 0.5
        c["rows"] = _log(rng, 1, 6000 if heads * c["dim"] <= 4096 else 3000)
        c["cached"], c["prefix"] = rng.choice([0, 0, _log(rng, 1, 2000)]), rng.choice([0, 0, _log(rng, 1, 1000)])
        c["seqs"] = _log(rng, 1, 32)
    else:
        c["op"], c["x"] = "attend8", rng.choice(["bf16", "f16"])
        c["dim"] = rng.choice([64, 128, 128, 128, 80, 96])
        if op == "prompt":
            c["form"] = "prompt"
            c["rows"] = min(_log(rng, 1, 4000), 96000 // heads)
            c["cached"], c["prefix"] = rng.choice([0, 0, _log(rng, 1, 3000)]), rng.choice([0, 0, _log(rng, 1, 1000)])
            c["seqs"] = _log(rng, 1, 8)
        else:
            c["form"] = "prefix"
            c["seqs"] = _log(rng, 1, 64)
            c["cached"] = _log(rng, 1, 12000 // kv_heads * 8 // max(8, c["seqs"] // 4))
            c["prefix"] = rng.choice([0, 0, _log(rng, 1, 2000)])
            each = rng.choice([1, 1, 1, 2, 5, 9])
            c["rows"] = c["seqs"] * each
            c["shortest"] = each if rng.random() < 0.5 else 0
            return c
    c["shortest"] = rng.choice([0, 1]) if c["rows"] >= c["seqs"] else 0
    return c


def _lengths(case):
    """Rows of each sequence (they add up to case["rows"], none below "shortest") and its cached positions, rows included."""
    r = random.Random(case["lens_seed"])
    B, T, lo = case["seqs"], case["rows"], case["shortest"]
    left = T - B * lo
    if B == 1 or left <= 0:
        n = [lo + (left if i == 0 else 0) for i in range(B)]
    elif case.get("form") == "prefix":
        n, most = [lo] * B, 2 * -(-T // B)                # a decoding batch: no sequence far over the others
        while left > 0:
            i = r.randrange(B)
            if n[i] < most:
                n[i] += 1
                left -= 1
    else:
        cuts = sorted(r.randrange(left + 1) for _ in range(B - 1))
        n = [lo + b - a for a, b in zip([0] + cuts, cuts + [left])]
    c = case["cached"]
    return n, [x + (r.randint(0, c) if B > 1 else c) for x in n]


# ----------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    s = _prepare_sample(case, g) if case["op"] == "sample" else _prepare_cache(case, g)
    s["case"] = case
    if own:
        import paper_2410_06916_b200 as lib
        s["lib"] = lib
        if case["op"] != "sample":
            s["batch"] = lib.RowBatch(lib.PagedKV(s["pool"], s["scales"]), s["row_start"], s["kv_len"], s["page_table"],
                                      n_rows=case["rows"], max_rows=max(1, max(s["n"])), prefix_pages=s["prefix_pages"],
                                      prefix_len=case["prefix"])
            s["out"] = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
        else:
            s["tokens"] = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
            s["probs"] = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    return s


def _prepare_sample(case, g):
    R, V = case["rows"], case["vocab"]
    x = torch.randn(R, V, generator=g, device="cuda") * case["spread"]
    # a model is sure of a few tokens: some dozen logits stand out, by an amount that varies from row to row
    few = torch.randint(0, V, (R, 12), generator=g, device="cuda")
    lift = torch.rand(R, 12, generator=g, device="cuda") * 6.0 * torch.rand(R, 1, generator=g, device="cuda")
    x.scatter_add_(1, few, lift)
    s = {"logits": x.to(DTYPES[case["dtype"]]), "uniforms": torch.rand(R, generator=g, device="cuda")}
    one = torch.ones(R, device="cuda")
    if case["mixed"]:
        kind = torch.randint(0, 6, (R,), generator=g, device="cuda")          # 0 greedy, 1 plain, 2 top-k, 3 top-p, 4 min-p, 5 all
        vary = 0.5 + torch.rand(R, generator=g, device="cuda")
        s["temperature"] = torch.where(kind == 0, 0.0, case["temperature"] * vary)
        s["top_k"] = torch.where((kind == 2) | (kind == 5), (case["k"] * vary).long(), 0).to(torch.int32)
        s["top_p"] = torch.where((kind == 3) | (kind == 5), one * case["p"], one)
        s["min_p"] = torch.where((kind == 4) | (kind == 5), one * case["min_p"], 0.0)
    else:
        s["temperature"], s["top_p"], s["min_p"] = one * case["temperature"], one * case["p"], one * case["min_p"]
        s["top_k"] = torch.full((R,), case["k"], dtype=torch.int32, device="cuda")
    return s


def _prepare_cache(case, g):
    dev = "cuda"
    B, T, H, Hk, D, P, blocks = case["seqs"], case["rows"], case["heads"], case["kv_heads"], case["dim"], case["page"], case["blocks"]
    n, kv = _lengths(case)
    per_seq = [-(-x // P) for x in kv]
    n_prefix = -(-case["prefix"] // P)
    n_pages = sum(per_seq) + n_prefix + 3
    perm = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    width = max(1, max(per_seq))
    table = torch.zeros(B, width, dtype=torch.int32)
    host = perm.cpu()
    at = n_prefix
    for i, m in enumerate(per_seq):
        table[i, :m] = host[at:at + m]
        at += m
    s = {"prefix_pages": perm[:n_prefix].contiguous(), "page_table": table.to(dev), "n": n, "kv": kv, "block": blocks - 1}
    # what earlier steps have left in the cache: K with dims of unlike size, V, each page and head by its own largest value
    shape = (n_pages, blocks, 2, Hk, P, D)
    unlike = torch.ones(2, Hk, 1, D, device=dev)
    unlike[0] = torch.exp(0.5 * torch.randn(Hk, 1, D, generator=g, device=dev))
    s["scales"] = torch.zeros(shape[:4], device=dev)
    s["pool"] = torch.zeros(shape, dtype=torch.uint8, device=dev).view(DTYPES[case["codes"]])
    step = max(1, (1 << 26) // (blocks * 2 * Hk * P * D))
    for p in range(0, n_pages, step):
        x = torch.randn((min(step, n_pages - p),) + shape[1:], generator=g, device=dev) * unlike
        top = x.abs().amax((-2, -1)) / LARGEST[case["codes"]]
        x = x / top[..., None, None]
        s["pool"][p:p + step] = (x.round() if case["codes"] == "i8" else x).to(DTYPES[case["codes"]])
        s["scales"][p:p + step] = top
    start = [0]
    for x in n:
        start.append(start[-1] + x)
    s["start"] = start
    s["row_start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    xt = DTYPES[case["x"]]
    # where every sequence's positions lie in the pool, as page * page_size + slot, and its rows in the packed tensors: the plan
    # of the plain form; what a sequence does not have is 0, and masked
    seq_page, own_pos = s["page_table"].long(), torch.arange(max(1, max(kv)), device=dev)
    own_at = seq_page[:, own_pos // P] * P + own_pos % P
    t = torch.arange(case["prefix"], device=dev)
    s["at"] = torch.cat([(s["prefix_pages"].long()[t // P] * P + t % P).expand(B, -1), own_at], 1)
    nt = torch.tensor(n, device=dev)
    most = torch.arange(max(1, max(n)), device=dev)
    s["real"] = most[None, :] < nt[:, None]                                    # [sequence, its row]
    s["row_of"] = torch.where(s["real"], s["row_start"][:-1, None] + most[None, :], 0)
    s["pos_of"] = torch.where(s["real"], (s["kv_len"] - nt)[:, None] + most[None, :], 0)
    s["padded"] = s["real"].reshape(-1).nonzero()[:, 0]
    s["rows"], s["pos"] = s["row_of"][s["real"]], s["pos_of"][s["real"]]         # every row in order, its own position
    if case["op"] == "append8":
        seq = s["real"].nonzero()[:, 0]
        s["page"] = seq_page[seq, s["pos"] // P]
        s["pages"] = s["page"].unique()                                         # those that get new positions
        s["earlier"] = torch.zeros(n_pages, dtype=torch.bool, device=dev)       # and those of them that had positions before
        s["earlier"][s["page"]] = s["pos"] // P * P < (s["kv_len"] - nt)[seq]
        x = torch.randn(T, (H + 2 * Hk) * D, generator=g, device=dev)           # the fused projection's rows
        x[:, H * D:(H + Hk) * D] *= unlike[0].reshape(1, -1)
        x = x.to(xt)
        s["q"] = x[:, :H * D].view(T, H, D)
        s["k"] = x[:, H * D:(H + Hk) * D].view(T, Hk, D)
        s["v"] = x[:, (H + Hk) * D:].view(T, Hk, D)
        s["gains"] = (1.0 + 0.1 * torch.randn(2, D, generator=g, device=dev)) if case["norm"] else None
        pairs = torch.arange(case["rotary_dim"] // 2, device=dev, dtype=torch.float64)
        freq = 10000.0 ** (-2.0 * pairs / case["rotary_dim"])
        ang = torch.arange(case["prefix"] + max(kv) + 1, device=dev, dtype=torch.float64)[:, None] * freq
        s["rope"] = torch.stack([ang.cos(), ang.sin()], dim=-1).float()          # the table that the program keeps
    else:
        s["q"] = torch.randn(T, H, D, generator=g, device=dev).to(xt)
    return s


# ----------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case = s["case"]
    if case["op"] == "sample":
        return s["lib"].sample_rows(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                    min_p=s["min_p"], tokens=s["tokens"], probs=s["probs"])
    b = s["batch"]
    if case["op"] == "append8":
        g = s["gains"]
        out = b.append(s["block"], s["q"], s["k"], s["v"], rope=s["rope"], interleaved=case["interleaved"],
                       q_gain=None if g is None else g[0], k_gain=None if g is None else g[1], eps=1e-5, out=s["out"])
        return out, s["pool"], s["scales"]
    return (b.prompt_attention if case["form"] == "prompt" else b.prefix_attention)(s["block"], s["q"], out=s["out"])


def _run_plain(s):
    op = s["case"]["op"]
    return _plain_sample(s) if op == "sample" else _plain_append(s) if op == "append8" else _plain_attention(s)


def _plain_append(s):
    """q in 32 bits, rounded once; K and V in 64, whose codes are then the nearest to their values: a value next to the border
    between two codes would else fall on either side."""
    case, P, b = s["case"], s["case"]["page"], s["block"]
    pool, scales, top = s["pool"], s["scales"], LARGEST[case["codes"]]
    rows, pos, page, pages = s["rows"], s["pos"], s["page"], s["pages"]
    cs = s["rope"][pos + case["prefix"]][:, None]
    half = case["rotary_dim"] // 2

    def finish(x, gain):
        c, sn = cs[..., 0].to(x.dtype), cs[..., 1].to(x.dtype)
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain.to(x.dtype)
        r, rest = x[..., :2 * half], x[..., 2 * half:]
        if case["interleaved"]:
            a, z = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * c - z * sn, z * c + a * sn], dim=-1).flatten(-2)
        else:
            a, z = r[..., :half], r[..., half:]
            r = torch.cat([a * c - z * sn, z * c + a * sn], dim=-1)
        return torch.cat([r, rest], dim=-1)

    gq, gk = (None, None) if s["gains"] is None else (s["gains"][0], s["gains"][1])
    q = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
    q[rows] = finish(s["q"][rows].float(), gq).to(q.dtype)
    x = torch.stack([finish(s["k"][rows].double(), gk), s["v"][rows].double()], 1)              # [row, K or V, kv head, dim]
    # the scale of each page: what its new values need, or what its earlier positions have where that is more
    amax = torch.zeros(pool.shape[0], *x.shape[1:3], dtype=torch.float64, device=x.device)
    amax.index_reduce_(0, page, x.abs().amax(-1), "amax")
    had = torch.where(s["earlier"][:, None, None], scales[:, b], 0.0)
    new = torch.maximum((amax / top).float(), had)
    ratio = torch.where(new > 0, had.double() / new.double(), 1.0)[pages]
    held = pool.view(torch.uint8)                                              # bytes: 8-bit floats are not indexed everywhere
    old = held[pages, b].view(pool.dtype).double()
    held[pages, b] = _code(old * ratio[..., None, None], pool.dtype).view(torch.uint8)
    scales[pages, b] = new[pages]
    inv = 1.0 / new[page].double()
    codes = _code(x * torch.where(inv.isinf(), 0.0, inv)[..., None], pool.dtype)
    held[page, b, :, :, pos % P] = codes.view(torch.uint8)
    return q, pool, scales


def _code(x, dtype):
    return x.round().to(dtype) if dtype == torch.int8 else x.float().to(dtype)


def _plain_attention(s):
    case, pool, P, b = s["case"], s["pool"], s["case"]["page"], s["block"]
    B, H, Hk, D, at = case["seqs"], case["heads"], case["kv_heads"], case["dim"], s["at"]
    G, L, n = H // Hk, s["at"].shape[1], s["row_of"].shape[1]
    codes = pool.view(torch.uint8)[at // P, b, :, :, at % P].view(pool.dtype).float()             # [B, L, K or V, kv head, dim]
    kv = (codes * s["scales"][at // P, b][..., None]).permute(2, 0, 3, 1, 4)                      # [K or V, B, kv head, L, dim]
    q = s["q"][s["row_of"]].float().view(B, n, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, D)
    a = torch.matmul(q, kv[0].transpose(-1, -2)).view(B, Hk, G, n, L).mul_(1.0 / math.sqrt(D))
    hidden = torch.arange(L, device=q.device) > (s["pos_of"] + case["prefix"])[..., None]         # [B, n, L]
    a.masked_fill_(hidden[:, None, None], float("-inf"))
    a.sub_(a.amax(-1, keepdim=True)).exp_()
    a.div_(a.sum(-1, keepdim=True))
    o = torch.matmul(a.view(B, Hk, G * n, L), kv[1]).view(B, Hk, G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    out = torch.zeros_like(s["q"])
    out[s["rows"]] = o.reshape(B * n, H, D)[s["padded"]].to(out.dtype)
    return out


def _plain_sample(s):
    """In 64 bits: the running sums are compared with a random number's share of their total."""
    x, u = s["logits"].float(), s["uniforms"].double()[:, None]
    V = x.shape[1]
    greedy = s["temperature"][:, None] == 0
    t = torch.where(greedy, 1.0, s["temperature"][:, None].double())
    by_size, order = x.sort(dim=1, descending=True, stable=True)                # among equals the lowest index first
    w = torch.exp((by_size.double() - by_size[:, :1].double()) / t)
    rank = torch.arange(V, device=x.device)[None, :]
    k = s["top_k"].long()[:, None]
    k = torch.where(greedy, 1, torch.where((k <= 0) | (k > V), V, k))
    w = torch.where(rank < k, w, 0.0)
    p = s["top_p"].double()[:, None]
    before = w.cumsum(1) - w
    keep = (rank < k) & ((p >= 1.0) | (before < p * w.sum(1, keepdim=True)) | (rank == 0)) & (w >= s["min_p"].double()[:, None])
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))        # back in the order of the vocabulary
    upto = w.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= u * total).sum(1, keepdim=True).clamp_(max=V - 1)
    return token[:, 0].to(torch.int32), (w.gather(1, token) / total)[:, 0].float()


# ----------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "sample":
        return _exact_sample(s)
    return _exact_append(s) if case["op"] == "append8" else _exact_attention(s)


def _exact_sample(s):
    probs = []
    for i in range(s["logits"].shape[0]):
        x = s["logits"][i].to(torch.float64)
        if s["temperature"][i] == 0:
            probs.append(torch.ones((), dtype=torch.float64, device=x.device))
            continue
        dist = torch.softmax(x / s["temperature"][i].to(torch.float64), 0)
        order = torch.argsort(-x, stable=True)
        if 0 < s["top_k"][i] < len(order):
            order = order[:int(s["top_k"][i])]
        if s["top_p"][i] < 1:
            share = torch.cumsum(dist[order], 0) / dist[order].sum()
            order = order[:1 + int((share < s["top_p"][i].to(torch.float64)).sum())]
        order = order[dist[order] >= s["min_p"][i].to(torch.float64) * dist[order[0]]]
        kept = torch.zeros_like(dist)
        kept[order] = dist[order] / dist[order].sum()
        at = torch.searchsorted(torch.cumsum(kept, 0), s["uniforms"][i].to(torch.float64), right=True)
        probs.append(kept[at])
    return None, torch.stack(probs)


def _exact_append(s):
    case, half, D = s["case"], s["case"]["rotary_dim"] // 2, s["case"]["dim"]
    q = s["q"].to(torch.float64).clone()
    if s["gains"] is not None:
        q *= s["gains"][0].to(torch.float64) / (q.square().sum(-1, keepdim=True) / D + 1e-5).sqrt()
    first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    for i in range(case["seqs"]):
        n, l, r0 = s["n"][i], s["kv"][i], s["start"][i]
        z = torch.view_as_complex(s["rope"][case["prefix"] + l - n:case["prefix"] + l].to(torch.float64))[:, None]
        w = torch.complex(q[r0:r0 + n, :, first], q[r0:r0 + n, :, second]) * z
        q[r0:r0 + n, :, first], q[r0:r0 + n, :, second] = w.real, w.imag
    return q, None, None


def _exact_attention(s):
    case, P, b = s["case"], s["case"]["page"], s["block"]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(case["rows"], H, D, dtype=torch.float64, device="cuda")
    for i in range(case["seqs"]):
        n, l, r0 = s["n"][i], s["kv"][i], s["start"][i]
        if n == 0:
            continue
        j, t = torch.arange(l, device="cuda"), torch.arange(case["prefix"], device="cuda")
        page = torch.cat([s["prefix_pages"].long()[t // P], s["page_table"][i].long()[j // P]])
        slot = torch.cat([t % P, j % P])
        N = len(page)
        seen = torch.ones(n, N, dtype=torch.bool, device="cuda").tril_(N - n)
        for h in range(Hk):
            code = s["pool"].view(torch.uint8)[page, b, :, h, slot].view(s["pool"].dtype).to(torch.float64)
            value = code * s["scales"][page, b, :, h].to(torch.float64)[..., None]                # [N, K or V, dim]
            for e in range(h * (H // Hk), (h + 1) * (H // Hk)):
                z = s["q"][r0:r0 + n, e].to(torch.float64) @ value[:, 0].T * D ** -0.5
                out[r0:r0 + n, e] = torch.softmax(torch.where(seen, z, -math.inf), -1) @ value[:, 1]
    return out


# ----------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "sample":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": case["rows"] * (case["vocab"] * size + 28), "flops": 4 * case["rows"] * case["vocab"]}
    n, kv = _lengths(case)
    H, Hk, D, T, P = case["heads"], case["kv_heads"], case["dim"], case["rows"], case["page"]
    size = 4 if case["x"] == "f32" else 2
    if case["op"] == "append8":
        seen = set()
        for a, l in zip(n, kv):
            seen.update(range(l - a, l))
        pages = sum((l - 1) // P - (l - a) // P + 1 for a, l in zip(n, kv) if a > 0)
        moved = T * (H + 2 * Hk) * D * size + T * H * D * size + T * 2 * Hk * D + pages * 2 * Hk * 4 + len(seen) * case["rotary_dim"] * 4
        return {"bytes": moved + (8 * D if case["norm"] else 0),
                "flops": T * (H + Hk) * (3 * case["rotary_dim"] + (4 * D if case["norm"] else 0)) + 4 * T * Hk * D}
    live = [(a, l) for a, l in zip(n, kv) if a > 0]
    pairs = sum(a * (case["prefix"] + l) - a * (a - 1) // 2 for a, l in live)
    cached = sum(l for _, l in live) + (case["prefix"] if live else 0)
    pages = sum(-(-l // P) for _, l in live) + (-(-case["prefix"] // P) if live else 0)
    return {"bytes": 2 * size * T * H * D + 2 * cached * Hk * D + pages * Hk * 8, "flops": 4 * pairs * H * D}
