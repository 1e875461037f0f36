"""Tokens drawn from logits against the definition in 64 bits: the token itself, unless the random number lies on a border."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
F64 = torch.float64


def reference(x, u, temperature=1.0, k=0, p=1.0, min_p=0.0):
    """(kept w by id, total) of one row on the host, or None for a row without an answer."""
    x = x.to(F64)
    V = len(x)
    if not (0 <= u < 1) or not (0 <= temperature < math.inf) or p != p or not (min_p <= 1):
        return None
    if x.isnan().any() or (x == math.inf).any() or (x == -math.inf).all():
        return None
    order = sorted(range(V), key=lambda i: (-float(x[i]), i)) if V < 3000 else torch.sort(x, descending=True, stable=True)[1].tolist()
    w = torch.zeros(V, dtype=F64)
    if temperature == 0:
        w[order[0]] = 1.0
        return w
    order = torch.tensor(order[:k] if 0 < k < V else order)
    e = torch.exp((x[order] - x[order[0]]) / temperature)
    if p < 1:
        upto = e.cumsum(0)
        keep = (upto - e) < p * upto[-1]
        keep[0] = True
        order, e = order[keep], e[keep]
    keep = e >= min_p
    w[order[keep]] = e[keep]
    return w


def check(logits, u, **kw):
    """Every row's token is the reference's, or one whose border u * total is nearer than the operator resolves: weights are rounded to
    2^-46 of the largest each, so a running sum over V tokens is off by at most V 2^-46, and so is the total; a cut of top-p that the
    same error decides changes sums by a weight more, which these inputs' rows avoid (their top-p border is checked below)."""
    from paper_2410_06916_b200 import sample_rows
    rows, V = logits.shape
    per_row = {n: (v if isinstance(v, torch.Tensor) else torch.full((rows,), v)) for n, v in
               (("temperature", kw.get("temperature", 1.0)), ("top_k", kw.get("top_k", 0)), ("top_p", kw.get("top_p", 1.0)), ("min_p", kw.get("min_p", 0.0)))}
    dev = {n: (v.cuda() if isinstance(v, torch.Tensor) else v) for n, v in kw.items()}
    tokens, probs = sample_rows(logits.cuda(), u.cuda(), **dev)
    tokens, probs = tokens.cpu(), probs.cpu()
    for r in range(rows):
        t, k, p, m = (per_row[n][r] for n in ("temperature", "top_k", "top_p", "min_p"))
        w = reference(logits[r], float(u[r]), float(t), int(k), float(p), float(m))
        if w is None:
            assert tokens[r] == -1 and probs[r] == 0
            continue
        upto = w.cumsum(0)
        goal, eps = float(u[r].to(F64)) * float(upto[-1]), 2 * V * 2.0 ** -46
        tok = int(tokens[r])
        assert 0 <= tok < V and w[tok] > 0, (r, tok)
        assert float(upto[tok] - w[tok]) <= goal + eps and float(upto[tok]) > goal - eps, (r, tok, goal)
        want = float(w[tok] / upto[-1])
        assert abs(float(probs[r]) - want) <= 2.0 ** -23 * want + 2 * V * 2.0 ** -46, (r, float(probs[r]), want)
    return tokens


def make(rows, V, spread=2.5, dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, V, generator=g) * spread).to(dtype), torch.rand(rows, generator=g)


@pytest.mark.parametrize("V", [1, 2, 31, 127, 129, 1000, 4097, 32000, 50257, 128256, 262144])
def test_plain_draws(V):
    check(*make(4, V, seed=V))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("kw", [dict(temperature=0.0), dict(temperature=0.7), dict(top_k=1), dict(top_k=50), dict(top_k=5000), dict(top_p=0.9),
                                dict(top_p=0.999, temperature=1.5), dict(min_p=0.05), dict(top_p=0.0), dict(min_p=1.0),
                                dict(temperature=0.8, top_k=100, top_p=0.9, min_p=0.02)], ids=str)
def test_filters(dtype, kw):
    check(*make(6, 20011, dtype=dtype, seed=3), **kw)


@pytest.mark.parametrize("kw", [dict(top_k=300), dict(top_p=0.5), dict(top_k=70000, top_p=0.7, min_p=0.3), dict(top_p=0.95, temperature=0.3)], ids=str)
def test_filters_large_vocabulary(kw):
    check(*make(3, 128000, dtype=torch.bfloat16, seed=4), **kw)
    check(*make(3, 151936, spread=0.3, seed=5), **kw)


def test_a_rows_settings_are_its_own():
    x, u = make(9, 3001, seed=6)
    check(x, u, temperature=torch.tensor([0, 1, 0.5, 2, 1, 1, 1e-3, 50, 1.0]), top_k=torch.tensor([0, 5, 3000, 3001, -7, 2, 40, 1 << 30, 1], dtype=torch.int32),
          top_p=torch.tensor([0.1, 1, 0.9, 0.3, 1e-9, 2.0, 0.5, 0.99, 0.5]), min_p=torch.tensor([0, 0, 0.1, 0, 0, 1.0, 0, 0.9, -3.0]))


def test_equal_logits_are_taken_in_the_order_of_ids():
    x = torch.zeros(5, 70000)
    x[1, 1000:] = 1.0
    x[2, ::7] = 2.0
    x[3] = -0.0
    x[3, ::2] = 0.0
    x[4, 30000:] = -math.inf
    u = torch.tensor([0.999, 0.5, 0.25, 0.9, 0.75])
    assert check(x, u, top_k=600).tolist() == [int(0.999 * 600), 1000 + 300, 7 * 150, 539, 450]       # (0.9 in fp32 is below 0.9)
    check(x, u, top_k=1000)
    check(x, u, top_p=0.26)
    assert check(x, u, temperature=0.0).tolist() == [0, 1000, 0, 0, 0]
    check(x.half(), u, top_k=69999, top_p=0.5)


def test_borders_of_the_running_sum():
    x = torch.zeros(6, 8)                                      # eight equal tokens: every border is exact
    u = torch.tensor([0.0, 0.125, 0.12499999, 0.5, 0.875, 1 - 2.0 ** -24])
    assert check(x, u).tolist() == [0, 1, 0, 4, 7, 7]
    assert check(x, u, top_p=0.5).tolist() == [0, 0, 0, 2, 3, 3]
    x[:, 0] = -math.inf                                        # an id that cannot be drawn
    assert check(x, u)[0] == 1


def test_rows_without_an_answer():
    x, u = make(14, 500, seed=8)
    x[0, 7], x[1, 499], x[2] = math.nan, math.inf, -math.inf
    u[3], u[4], u[5] = 1.0, -0.1, math.nan
    t, p, m = torch.ones(14), torch.ones(14), torch.zeros(14)
    t[6], t[7], t[8], p[9], m[10], m[11] = -1.0, math.inf, math.nan, math.nan, math.nan, 1.5
    x[12, 3] = -math.nan
    got = check(x, u, temperature=t, top_p=p, min_p=m)
    assert (got[:13] == -1).all() and got[13] >= 0
    got = check(x, u, temperature=torch.zeros(14))             # greedy rows are checked as well
    assert got[:6].tolist() == [-1] * 6 and got[6] >= 0


def test_extreme_temperatures_and_logits():
    x, u = make(4, 4000, seed=9)
    check(x, u, temperature=1e-38, top_p=0.5)
    check(x, u, temperature=3e38, top_p=0.5, top_k=100)
    check(x * 1e37, u, top_k=10, top_p=0.9)
    check(x * 1e-40, u, top_k=10, top_p=0.9)


def test_rows_of_a_wider_tensor_and_odd_starts():
    wide, u = make(5, 5001, seed=10)
    for cut in (slice(0, 4000), slice(1, 4002), slice(3, 3)):
        if wide[:, cut].shape[1]:
            check(wide[:, cut], u, top_k=40)
            check(wide.bfloat16()[:, cut], u, top_p=0.8)
    from paper_2410_06916_b200 import sample_rows
    d = wide.cuda()
    a = sample_rows(d[:, 1:4002], u.cuda(), top_p=0.9)
    b = sample_rows(d[:, 1:4002].contiguous(), u.cuda(), top_p=0.9)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_rows_token_does_not_depend_on_the_batch():
    """One row alone is spread over more blocks than a row of a large batch."""
    from paper_2410_06916_b200 import sample_rows
    x, u = make(300, 12000, seed=11)
    x, u = x.cuda(), u.cuda()
    for kw in (dict(), dict(top_p=0.9), dict(top_k=77, top_p=0.8)):
        tokens, probs = sample_rows(x, u, **kw)
        for r in (0, 17, 299):
            t, q = sample_rows(x[r:r + 1], u[r:r + 1], **kw)
            assert t[0] == tokens[r] and q[0] == probs[r]


@pytest.mark.parametrize("V", [5000, 12000, 20000, 40000, 128000])
def test_the_same_call_gives_the_same_bits(V):
    from paper_2410_06916_b200 import sample_rows
    x, u = make(300, V, seed=20 + V)
    x, u = x.cuda(), u.cuda()
    for kw in (dict(top_p=0.9), dict(top_k=77, top_p=0.8), dict(top_k=500), dict()):
        want = sample_rows(x, u, **kw)
        for _ in range(30):
            got = sample_rows(x, u, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_draws_follow_the_distribution():
    """20000 draws from one row: each token's count within five standard deviations of what its probability says."""
    from paper_2410_06916_b200 import sample_rows
    g = torch.Generator().manual_seed(12)
    x = torch.randn(1, 40, generator=g)
    n = 20000
    u = torch.rand(n, generator=g)
    tokens, _ = sample_rows(x.expand(n, 40).contiguous().cuda(), u.cuda(), temperature=0.8, top_k=30, top_p=0.95)
    w = reference(x[0], 0.5, 0.8, 30, 0.95)
    pr = w / w.sum()
    count = torch.bincount(tokens.cpu().long(), minlength=40).to(F64)
    assert ((count - n * pr).abs() <= 5 * (n * pr * (1 - pr)).sqrt() + 1e-9).all()


def test_a_captured_call_follows_its_inputs():
    from paper_2410_06916_b200 import sample_rows
    x, u = (t.cuda() for t in make(4, 9000, seed=13))
    k = torch.full((4,), 20, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sample_rows(x, u, top_k=k)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens, probs = sample_rows(x, u, top_k=k, top_p=0.9)
    for seed in (14, 15):
        y, v = make(4, 9000, seed=seed)
        x.copy_(y), u.copy_(v), k.fill_(seed)
        graph.replay()
        want = sample_rows(x, u, top_k=k, top_p=0.9)
        assert torch.equal(tokens, want[0]) and torch.equal(probs, want[1])


def test_outputs_and_streams():
    from paper_2410_06916_b200 import sample_rows
    x, u = (t.cuda() for t in make(4, 3000, seed=16))
    tokens, probs = torch.full((6,), 7, dtype=torch.int32, device="cuda"), torch.full((6,), 7.0, device="cuda")
    want = sample_rows(x, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sample_rows(x, u, tokens=tokens[1:5], probs=probs[1:5], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert got[0].data_ptr() == tokens[1:].data_ptr()
    assert torch.equal(tokens[1:5], want[0]) and torch.equal(probs[1:5], want[1])
    assert tokens[0] == 7 and tokens[5] == 7 and probs[0] == 7 and probs[5] == 7
    empty = sample_rows(x[:0], u[:0])
    assert empty[0].shape == (0,)
