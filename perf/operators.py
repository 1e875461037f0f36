"""The operators for batches of sequences over a paged K,V cache: what is measured, and on what.

Four operators, as a serving program chains them in every layer:
  rope      cos/sin table of the rotary positions, plain or scaled for long contexts
  append    per-head norm of q and k, rotation, and K,V into the pages of the cache, in one pass
  prompt    causal attention over whole prompts (or chunks of them), grouped heads, packed ragged sequences
  prefix    attention of a few rows per sequence, behind a prefix that all sequences share

The cache is one pool [page][block][K or V][kv head][slot][dim] for all layers, the layout of the library's own cache.
`own = False` computes them from elementary torch operations in 32 bits; `own = True` calls the library.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ----------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a table for the context lengths of the 7B and 13B shapes, made at start-up
        {"name": "rope 4k", "op": "rope", "positions": 4096, "rotary_dim": 128, "theta": 10000.0, "factor": 1.0, "original": 0,
         "low": 1.0, "high": 4.0},
        # a table stretched by parts to a long context, a quarter of the head rotated
        {"name": "rope 200k by parts", "op": "rope", "positions": 200001, "rotary_dim": 128, "theta": 500000.0, "factor": 8.0,
         "original": 8192, "low": 1.0, "high": 4.0},
        # one decoding step of 16 sequences of the 13B shape: a token each; latency counts
        {"name": "append decode 13b", "op": "append", "dtype": "bf16", "x": "bf16", "heads": 40, "kv_heads": 40, "dim": 128,
         "page": 16, "seqs": 16, "rows": 16, "shortest": 1, "cached": 1000, "prefix": 0, "lens_seed": 1, "rotary_dim": 128,
         "interleaved": False, "norm": False, "blocks": 2},
        # the prompts of a batch of the 70B shape with normed queries and keys, out of the fused projection
        {"name": "append prompts 70b", "op": "append", "dtype": "bf16", "x": "bf16", "heads": 64, "kv_heads": 8, "dim": 128,
         "page": 16, "seqs": 7, "rows": 8192, "shortest": 100, "cached": 0, "prefix": 0, "lens_seed": 2, "rotary_dim": 128,
         "interleaved": False, "norm": True, "blocks": 2},
        # neighbouring pairs over half of a small head, fp32 activations into an fp16 cache, continuing cached prompts
        {"name": "append pairs f16", "op": "append", "dtype": "f16", "x": "f32", "heads": 24, "kv_heads": 6, "dim": 64,
         "page": 32, "seqs": 5, "rows": 3001, "shortest": 0, "cached": 700, "prefix": 333, "lens_seed": 3, "rotary_dim": 32,
         "interleaved": True, "norm": True, "blocks": 1},
        # one 512-token prompt of the 7B shape (config 2)
        {"name": "prompt 512 7b", "op": "prompt", "dtype": "bf16", "heads": 32, "kv_heads": 32, "dim": 128, "page": 16,
         "seqs": 1, "rows": 512, "shortest": 512, "cached": 0, "prefix": 0, "lens_seed": 1, "blocks": 1},
        # ragged prompts of the 34B shape (seven query heads on a KV head), some continuing what is cached
        {"name": "prompt ragged 34b", "op": "prompt", "dtype": "f16", "heads": 56, "kv_heads": 8, "dim": 128, "page": 32,
         "seqs": 9, "rows": 5003, "shortest": 1, "cached": 600, "prefix": 0, "lens_seed": 4, "blocks": 2},
        # one long prompt of the 70B shape
        {"name": "prompt 8k 70b", "op": "prompt", "dtype": "bf16", "heads": 64, "kv_heads": 8, "dim": 128, "page": 64,
         "seqs": 1, "rows": 8192, "shortest": 8192, "cached": 0, "prefix": 0, "lens_seed": 1, "blocks": 1},
        # two sequences, a token each, heads of 64: the smallest decoding step
        {"name": "prefix smallest", "op": "prefix", "dtype": "bf16", "heads": 4, "kv_heads": 4, "dim": 64, "page": 16,
         "seqs": 2, "rows": 2, "shortest": 1, "cached": 60, "prefix": 100, "lens_seed": 1, "blocks": 1},
        # 33 candidates re-predicting a window of 32 tokens behind a 1024-token prompt (config 3's scoring at the 13B shape)
        {"name": "prefix candidates 13b", "op": "prefix", "dtype": "bf16", "heads": 40, "kv_heads": 40, "dim": 128, "page": 16,
         "seqs": 33, "rows": 1056, "shortest": 32, "cached": 0, "prefix": 1024, "lens_seed": 1, "blocks": 1},
        # 64 continuations of one long prompt of the 70B shape, a token each
        {"name": "prefix 64 of 70b", "op": "prefix", "dtype": "bf16", "heads": 64, "kv_heads": 8, "dim": 128, "page": 16,
         "seqs": 64, "rows": 64, "shortest": 1, "cached": 1500, "prefix": 8192, "lens_seed": 2, "blocks": 1},
        # verification of 8 drafts on each of 12 sequences of the 34B shape, ragged, a short shared system prompt
        {"name": "prefix verify 34b", "op": "prefix", "dtype": "f16", "heads": 56, "kv_heads": 8, "dim": 128, "page": 32,
         "seqs": 12, "rows": 108, "shortest": 9, "cached": 2500, "prefix": 301, "lens_seed": 5, "blocks": 1},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "append", "prompt", "prompt", "prompt", "prefix", "prefix", "prefix"])
    if op == "rope":
        original = rng.choice([0, 0, 2048, 8192, 32768])
        return {"op": op, "positions": _log(rng, 1, 200000), "rotary_dim": rng.choice([16, 32, 64, 80, 96, 128]),
                "theta": rng.choice([10000.0, 500000.0, 1000000.0]), "factor": rng.choice([1.0, 2.0, 4.0, 8.0, 32.0]),
                "original": original, "low": 1.0, "high": rng.choice([4.0, 32.0])}
    heads, kv_heads = rng.choice([(32, 32), (40, 40), (64, 8), (56, 8), (32, 8), (16, 2), (4, 4), (12, 1), (8, 4), (9, 3)])
    c = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "heads": heads, "kv_heads": kv_heads, "page": rng.choice([8, 16, 32, 64, 128]),
         "lens_seed": rng.randrange(1 << 20), "blocks": rng.choice([1, 2])}
    if op == "append":
        c["dim"] = rng.choice([16, 64, 80, 96, 128, 256])
        c["rotary_dim"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2])
        c["x"] = rng.choice([c["dtype"], "f32"])
        c["interleaved"], c["norm"] = rng.random() < 0.4, rng.random() < 0.5
        c["rows"] = _log(rng, 1, 6000)
        c["cached"], c["prefix"] = rng.choice([0, 0, _log(rng, 1, 2000)]), rng.choice([0, 0, _log(rng, 1, 1000)])
        most = 32
    elif op == "prompt":
        c["dim"] = rng.choice([64, 128, 128, 128, 80, 96])
        c["rows"] = min(_log(rng, 1, 8000), 512000 // heads)
        c["cached"], c["prefix"] = rng.choice([0, 0, _log(rng, 1, 1500)]), rng.choice([0, 0, _log(rng, 1, 1000)])
        most = 16
    else:
        c["dim"] = rng.choice([64, 128, 128, 128, 80, 96])
        c["cached"], c["prefix"] = _log(rng, 1, 3000), rng.choice([0, _log(rng, 1, 8000), _log(rng, 64, 8000)])
        most = 64
    c["seqs"] = _log(rng, 1, most)
    if op == "prefix":
        each = rng.choice([1, 1, 2, 5, 9, 16, 32])
        c["rows"] = c["seqs"] * each
        c["shortest"] = each if rng.random() < 0.5 else 0
    else:
        c["shortest"] = rng.choice([0, 1]) if c["rows"] >= c["seqs"] else 0
    return c


def _lengths(case):
    """Rows of each sequence (they add up to case["rows"], none below "shortest") and its cached positions, rows included."""
    r = random.Random(case["lens_seed"])
    B, T, lo = case["seqs"], case["rows"], case["shortest"]
    left = T - B * lo
    if B == 1 or left <= 0:
        n = [lo + (left if i == 0 else 0) for i in range(B)]
    elif case["op"] == "prefix":
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
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    dev = "cuda"
    s = {"case": case}
    if case["op"] == "rope":
        # the spread of the angles is an input too: theta and the factor move a little with the seed
        u = torch.rand(2, generator=g, device=dev, dtype=torch.float64).tolist()
        s["theta"] = case["theta"] * (1.0 + 0.01 * u[0])
        s["factor"] = case["factor"] * (1.0 + (0.01 * u[1] if case["factor"] != 1.0 else 0.0))
        s["magnitude"] = 0.1 * math.log(s["factor"]) + 1.0 if s["factor"] > 1.0 else 1.0
        if own:
            import paper_2410_06916_b200 as lib
            s["out"] = torch.empty(case["positions"], case["rotary_dim"] // 2, 2, device=dev)
            s["lib"] = lib
        return s
    dt = DTYPES[case["dtype"]]
    B, T, H, Hk, D, P = case["seqs"], case["rows"], case["heads"], case["kv_heads"], case["dim"], case["page"]
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
    s["pool"] = torch.randn(n_pages, case["blocks"], 2, Hk, P, D, generator=g, device=dev).to(dt)
    s["prefix_pages"] = perm[:n_prefix].contiguous()
    s["page_table"] = table.to(dev)
    s["n"], s["kv"] = n, kv
    start = [0]
    for x in n:
        start.append(start[-1] + x)
    s["start"] = start
    s["row_start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    s["block"] = case["blocks"] - 1
    if case["op"] == "append":
        xt = DTYPES[case["x"]]
        x = torch.randn(T, (H + 2 * Hk) * D, generator=g, device=dev).to(xt)      # the fused projection's rows
        s["q"] = x[:, :H * D].view(T, H, D)
        s["k"] = x[:, H * D:(H + Hk) * D].view(T, Hk, D)
        s["v"] = x[:, (H + Hk) * D:].view(T, Hk, D)
        s["gains"] = (1.0 + 0.1 * torch.randn(2, D, generator=g, device=dev)) if case["norm"] else None
        s["positions"] = case["prefix"] + max(kv) + 1
    else:
        s["q"] = torch.randn(T, H, D, generator=g, device=dev).to(dt)
    if own:
        import paper_2410_06916_b200 as lib
        s["batch"] = lib.RowBatch(lib.PagedKV(s["pool"]), s["row_start"], s["kv_len"], s["page_table"], n_rows=T,
                                  max_rows=max(1, max(n)), prefix_pages=s["prefix_pages"], prefix_len=case["prefix"])
        if case["op"] == "append":
            s["rope"] = lib.rope_table(s["positions"], case["rotary_dim"])
        s["out"] = torch.empty(T, H, D, device=dev, dtype=dt)
    else:
        if case["op"] == "append":
            pos = torch.arange(s["positions"], device=dev, dtype=torch.float64)
            ang = pos[:, None] * _frequencies(case["rotary_dim"], 10000.0, 1.0, 0, 1.0, 4.0)[None, :]
            s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        # where every sequence's positions lie in the pool, as page * page_size + slot: the plan of the plain form
        def slots(pages, length):
            p = torch.arange(length, device=dev)
            return pages.long()[p // P] * P + p % P
        s["prefix_slots"] = slots(s["prefix_pages"], case["prefix"])
        s["slots"] = [slots(s["page_table"][i], kv[i]) for i in range(B)]
    return s


def _frequencies(rotary_dim, theta, factor, original, low, high):
    """Angle per position of each pair, in 64 bits: theta^(-2i/rotary_dim), those of long wavelengths divided by the factor."""
    i = torch.arange(rotary_dim // 2, device="cuda", dtype=torch.float64)
    f = theta ** (-2.0 * i / rotary_dim)
    if original > 0:
        turns = original * f / (2.0 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0.0, 1.0)
    else:
        keep = torch.zeros_like(f)
    return (1.0 - keep) * f / factor + keep * f


# ----------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case = s["case"]
    op = case["op"]
    if op == "rope":
        return s["lib"].rope_table(case["positions"], case["rotary_dim"], theta=s["theta"], factor=s["factor"],
                                   original_positions=case["original"], low_turns=case["low"], high_turns=case["high"],
                                   magnitude=s["magnitude"], out=s["out"])
    b = s["batch"]
    if op == "append":
        g = s["gains"]
        out = b.append(s["block"], s["q"], s["k"], s["v"], rope=s["rope"], interleaved=case["interleaved"],
                       q_gain=None if g is None else g[0], k_gain=None if g is None else g[1], eps=1e-5, out=s["out"])
        return out, s["pool"]
    if op == "prompt":
        return b.prompt_attention(s["block"], s["q"], out=s["out"])
    return b.prefix_attention(s["block"], s["q"], out=s["out"])


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "rope":
        f = _frequencies(case["rotary_dim"], s["theta"], s["factor"], case["original"], case["low"], case["high"])
        ang = torch.arange(case["positions"], device="cuda", dtype=torch.float64)[:, None] * f[None, :]
        return (torch.stack([ang.cos(), ang.sin()], dim=-1) * s["magnitude"]).float()
    if op == "append":
        return _plain_append(s, case)
    return _plain_attention(s, case)


def _plain_append(s, case):
    pos = torch.cat([torch.arange(l - n, l, device="cuda") for n, l in zip(s["n"], s["kv"])]) + case["prefix"]
    c, sn = s["cos"][pos][:, None, :], s["sin"][pos][:, None, :]
    q, k, v = s["q"].float(), s["k"].float(), s["v"]
    if s["gains"] is not None:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-5) * s["gains"][0]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-5) * s["gains"][1]
    half = case["rotary_dim"] // 2

    def rotate(x):
        r, rest = x[..., :2 * half], x[..., 2 * half:]
        if case["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            r = torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)
        return torch.cat([r, rest], dim=-1)

    pool = s["pool"]
    slots = torch.cat([x[l - n:] for x, n, l in zip(s["slots"], s["n"], s["kv"])])
    page, slot = slots // case["page"], slots % case["page"]
    pool[page, s["block"], 0, :, slot] = rotate(k).to(pool.dtype)
    pool[page, s["block"], 1, :, slot] = v.to(pool.dtype)
    return rotate(q).to(pool.dtype), pool


def _plain_attention(s, case):
    q, pool, P, b = s["q"], s["pool"], case["page"], s["block"]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    G = H // Hk
    out = torch.zeros_like(q)
    for i in range(case["seqs"]):
        n, l = s["n"][i], s["kv"][i]
        if n == 0:
            continue
        at = torch.cat([s["prefix_slots"], s["slots"][i]])
        k = pool[at // P, b, 0, :, at % P].float().transpose(0, 1)           # [kv heads, positions, dim]
        v = pool[at // P, b, 1, :, at % P].float().transpose(0, 1)
        N = case["prefix"] + l
        key = torch.arange(N, device="cuda")
        step = max(1, (1 << 28) // (H * N))                                   # rows at a time: the scores stay near 1 GB
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            x = q[s["start"][i] + r0:s["start"][i] + r1].float().view(r1 - r0, Hk, G, D).permute(1, 2, 0, 3).reshape(Hk, G * (r1 - r0), D)
            a = torch.bmm(x, k.transpose(1, 2)) / math.sqrt(D)
            last = torch.arange(r0, r1, device="cuda") + (N - n)
            a = a.view(Hk, G, r1 - r0, N).masked_fill_(key[None, :] > last[:, None], float("-inf"))
            a = a - a.amax(-1, keepdim=True)
            a = a.exp_()
            a = a / a.sum(-1, keepdim=True)
            o = torch.bmm(a.view(Hk, G * (r1 - r0), N), v).view(Hk, G, r1 - r0, D).permute(2, 0, 1, 3).reshape(r1 - r0, H, D)
            out[s["start"][i] + r0:s["start"][i] + r1] = o.to(q.dtype)
    return out


# ----------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64 = torch.float64
    if case["op"] == "rope":
        half = case["rotary_dim"] // 2
        freq = []
        for i in range(half):
            f = s["theta"] ** (-i / half)
            t = 0.0
            if case["original"]:
                t = min(1.0, max(0.0, (case["original"] * f / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])))
            freq.append(f * (t + (1.0 - t) / s["factor"]))
        ang = torch.outer(torch.arange(case["positions"], dtype=f64, device="cuda"), torch.tensor(freq, dtype=f64, device="cuda"))
        z = torch.polar(torch.full_like(ang, s["magnitude"]), ang)
        return torch.view_as_real(z)
    P, b, D = case["page"], s["block"], case["dim"]
    if case["op"] == "append":
        half = case["rotary_dim"] // 2
        f = torch.tensor([10000.0 ** (-i / half) for i in range(half)], dtype=f64, device="cuda")
        pool, q = s["pool"].to(f64), s["q"].to(f64).clone()
        k = s["k"].to(f64).clone()
        if s["gains"] is not None:
            for x, g in ((q, s["gains"][0]), (k, s["gains"][1])):
                x *= g.to(f64) / (x.square().sum(-1, keepdim=True) / D + 1e-5).sqrt()
        first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else half)
        for i in range(case["seqs"]):
            n, l, r0 = s["n"][i], s["kv"][i], s["start"][i]
            if n == 0:
                continue
            z = torch.polar(torch.ones(n, half, dtype=f64, device="cuda"),
                            torch.outer(torch.arange(l - n, l, dtype=f64, device="cuda") + case["prefix"], f))[:, None]
            for x in (q, k):
                w = torch.complex(x[r0:r0 + n, :, first], x[r0:r0 + n, :, second]) * z
                x[r0:r0 + n, :, first], x[r0:r0 + n, :, second] = w.real, w.imag
            j = torch.arange(l - n, l, device="cuda")
            page = s["page_table"][i].long()[j // P]
            pool[page, b, 0, :, j % P] = k[r0:r0 + n]
            pool[page, b, 1, :, j % P] = s["v"][r0:r0 + n].to(f64)
        return q, pool
    H, Hk = case["heads"], case["kv_heads"]
    out = torch.zeros(case["rows"], H, D, dtype=f64, device="cuda")
    for i in range(case["seqs"]):
        n, l, r0 = s["n"][i], s["kv"][i], s["start"][i]
        if n == 0:
            continue
        j = torch.arange(l, device="cuda")
        t = torch.arange(case["prefix"], device="cuda")
        page = torch.cat([s["prefix_pages"].long()[t // P], s["page_table"][i].long()[j // P]])
        slot = torch.cat([t % P, j % P])
        N = len(page)
        seen = torch.ones(n, N, dtype=torch.bool, device="cuda").tril_(N - n)
        for h in range(H):
            K, V = pool_rows(s, page, slot, b, h // (H // Hk))
            z = s["q"][r0:r0 + n, h].to(f64) @ K.T * D ** -0.5
            z = torch.where(seen, z, -math.inf)
            out[r0:r0 + n, h] = torch.softmax(z, -1) @ V
    return out


def pool_rows(s, page, slot, block, head):
    x = s["pool"][page, block, :, head, slot].to(torch.float64)
    return x[:, 0], x[:, 1]


# ----------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "rope":
        pairs = case["positions"] * (case["rotary_dim"] // 2)
        return {"bytes": 8 * pairs, "flops": 6 * pairs}
    n, kv = _lengths(case)
    H, Hk, D, T = case["heads"], case["kv_heads"], case["dim"], case["rows"]
    if case["op"] == "append":
        size = 4 if case["x"] == "f32" else 2
        seen = set()
        for a, l in zip(n, kv):
            seen.update(range(l - a, l))
        moved = T * (H + 2 * Hk) * D * (size + 2) + len(seen) * case["rotary_dim"] * 4 + (8 * D if case["norm"] else 0)
        return {"bytes": moved, "flops": T * (H + Hk) * (3 * case["rotary_dim"] + (4 * D if case["norm"] else 0))}
    live = [(a, l) for a, l in zip(n, kv) if a > 0]
    pairs = sum(a * (case["prefix"] + l) - a * (a - 1) // 2 for a, l in live)
    cached = sum(l for _, l in live) + (case["prefix"] if live else 0)
    return {"bytes": 2 * (2 * T * H * D + 2 * cached * Hk * D), "flops": 4 * pairs * H * D}
