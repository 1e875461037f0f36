"""The operators over an 8-bit paged cache on the GPU against their 64-bit definitions (tests/paged8_reference.py derives the bounds)."""
import pytest
import torch

from paged_reference import F64, finish_heads, frequencies, append_tolerance
from paged8_reference import E4M3, I8, LARGEST, Batch8, append8, as_codes, attention8

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def setup(b: Batch8, **more):
    from paper_2410_06916_b200 import PagedKV, RowBatch
    args, kw = b.device_args()
    kw.update(more)
    pool, scales = b.pool.cuda(), b.scales.cuda()
    return pool, scales, RowBatch(PagedKV(pool, scales), *args, **kw)


def close(got, want, tol):
    got, want, tol = got.to(F64).cpu(), want.cpu(), tol.cpu()
    assert torch.isfinite(got).all()
    off = (got - want).abs() - tol
    assert (off <= 0).all(), f"{int((off > 0).sum())} of {off.numel()} outside; worst {float(off.max())} over, at {(off == off.max()).nonzero()[0].tolist()}"


# ----------------------------------------------------------------------------------------------- append
def rows_of(b, R, norm, strided=True, seed=5, grow=None):
    """q, k, v as slices of a fused projection, the gains and the rotary table, on the host."""
    H, Hk, D, T = b.heads, b.kv_heads, b.dim, b.n_rows
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, (H + 2 * Hk) * D + (16 if strided else 0), generator=g)
    if grow is not None:
        x *= grow
    x = x.to(b.x)
    gains = (1 + 0.2 * torch.randn(2, D, generator=g)) if norm else None
    longest = b.prefix_len + max(b.kv + [0]) + 1
    ang = torch.outer(torch.arange(longest, dtype=F64), torch.tensor(frequencies(R), dtype=F64)) if R else None
    table = torch.stack([ang.cos(), ang.sin()], -1).float() if R else None
    cut = lambda y: (y[:, :H * D].view(T, H, D), y[:, H * D:(H + Hk) * D].view(T, Hk, D), y[:, (H + Hk) * D:(H + 2 * Hk) * D].view(T, Hk, D))
    return x, cut, gains, table


def check_append(b: Batch8, R, interleaved, norm, positions=None, strided=True, eps=1e-5, grow=None, pool=None):
    pool, scales, batch = setup(b)
    x, cut, gains, table = rows_of(b, R, norm, strided, grow=grow)
    q, k, v = cut(x)
    qd, kd, vd = cut(x.cuda())
    out = torch.full((b.n_rows, b.heads, b.dim), 3.0, device="cuda", dtype=b.x)
    gd = gains.cuda() if norm else None
    got = batch.append(b.block, qd, kd, vd, rope=None if table is None else table.cuda(), interleaved=interleaved,
                       q_gain=gd[0] if norm else None, k_gain=gd[1] if norm else None, eps=eps,
                       positions=None if positions is None else positions.cuda(), out=out)
    assert got.data_ptr() == out.data_ptr()
    want, want_scales, near = append8(b, b.pool, b.scales, k, v, table, interleaved, gains[1] if norm else None, eps, positions)
    same = lambda a, c: (a == c) | (a.isnan() & c.isnan())
    assert same(scales.cpu(), want_scales).all()
    code = pool.cpu().to(F64)
    assert (same(code, want) | (near & ((code - want).abs() <= 1))).all()
    # q: rows that are left out keep what out held
    want_q, tol = torch.full((b.n_rows, b.heads, b.dim), 3.0, dtype=F64), torch.zeros(b.n_rows, b.heads, b.dim, dtype=F64)
    for i, n in enumerate(b.n):
        own = torch.arange(n) + b.kv[i] - n
        rows = torch.arange(n) + b.start[i]
        keep = (own >= 0) & (own < b.page_table.shape[1] * b.page)
        own, rows = own[keep], rows[keep]
        if not len(own):
            continue
        pages = b.page_table[i].long()[own // b.page]
        pos = own + b.prefix_len if positions is None else positions[rows].long()
        keep = (pages >= 0) & (pages < b.n_pages)
        if R:
            keep &= (pos >= 0) & (pos < table.shape[0])
        y, mag = finish_heads(q[rows[keep]], pos[keep], frequencies(R) if R else None, interleaved, gains[0] if norm else None, eps)
        want_q[rows[keep]], tol[rows[keep]] = y, append_tolerance(y, mag, b.dim, b.x)
    fine = want_q.isfinite() & (want_q.abs() < 1e37)         # (a row of infinities has a q of its own)
    close(torch.where(fine, out.to(F64).cpu(), 0.0), torch.where(fine, want_q, 0.0), torch.where(fine, tol, 0.0))


APPEND = [
    # rows, cached, heads, kv heads, dim, page, codes, x type, rotary dims, pairs side by side, norm
    ([1], [1], 4, 4, 64, 16, I8, BF16, 64, False, False),
    ([5, 0, 1, 40], [5, 7, 33, 45], 8, 2, 128, 16, I8, BF16, 128, False, True),
    ([5, 0, 1, 40], [5, 7, 33, 45], 8, 2, 128, 16, E4M3, F16, 128, False, True),
    ([3, 17], [20, 17], 7, 1, 128, 8, I8, F32, 128, True, True),
    ([9] * 33, [9 + i for i in range(33)], 4, 2, 64, 32, E4M3, F32, 32, False, False),
    ([2] * 70, [2 + 3 * i for i in range(70)], 2, 2, 16, 8, I8, F32, 16, False, True),
    ([13, 4], [13, 4], 3, 3, 80, 64, I8, F16, 32, True, True),
    ([13, 4], [13, 4], 3, 3, 80, 64, E4M3, BF16, 80, False, True),
    ([6, 2], [6, 9], 2, 1, 256, 128, I8, BF16, 128, False, True),
    ([150, 300], [150, 333], 2, 2, 128, 128, I8, BF16, 128, False, False),
    ([6, 2], [6, 9], 4, 2, 96, 16, I8, BF16, 0, False, True),         # no rotation
    ([6, 2], [6, 9], 5, 5, 34, 16, I8, F32, 10, False, True),         # dims and rotated dims of no particular size
    ([6, 2], [6, 9], 5, 1, 50, 16, E4M3, F16, 50, True, False),
    ([4, 3], [2, 1], 2, 2, 64, 16, I8, BF16, 64, False, False),       # more rows than cached positions: the first are left out
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c[2:]))
def test_append(case):
    n, kv, H, Hk, D, page, codes, xt, R, inter, norm = case
    check_append(Batch8(n, kv, H, Hk, D, page, codes, xt, padding=3, blocks=2, block=1), R, inter, norm)


@pytest.mark.parametrize("codes", [I8, E4M3], ids=str)
@pytest.mark.parametrize("factor", [0.01, 30.0])
def test_append_to_pages_with_earlier_positions(codes, factor):
    """Rows far smaller than what a page holds keep its scale; far larger ones have its codes rounded anew."""
    check_append(Batch8([1, 3, 20], [8, 20, 37], 2, 2, 64, 16, codes, spread=2.0), 64, False, False, grow=factor)


def test_append_behind_a_prefix_and_at_given_positions():
    b = Batch8([4, 2, 5], [11, 2, 70], 4, 2, 128, 16, I8, prefix_len=21)
    check_append(b, 128, False, True)
    depth = torch.tensor([7, 8, 8, 9, 21, 22, 0, 1000000, -1, 60, 61], dtype=torch.int32)   # two of them outside the table
    check_append(b, 128, False, False, positions=depth)
    check_append(Batch8([20], [20], 2, 2, 64, 16, E4M3), 64, False, False,                  # pages that start afresh, all or some rows left out
                 positions=torch.tensor([-1] * 16 + [0, -1, 2, 1 << 20], dtype=torch.int32))


def test_append_leaves_out_rows_whose_page_is_outside_the_pool():
    b = Batch8([4, 20], [20, 20], 4, 2, 64, 8, I8, blocks=2)
    b.page_table[1, 1] = -5
    b.page_table[1, 2] = b.n_pages
    b.page_table[0, 2] = 1 << 30
    check_append(b, 64, False, True)


def test_append_leaves_out_rows_behind_the_page_table():
    b = Batch8([20, 3], [40, 3], 4, 2, 64, 8, I8)
    b.page_table = b.page_table[:, :4].contiguous()        # the first sequence's last eight positions have no page
    check_append(b, 64, False, False)


@pytest.mark.parametrize("codes", [I8, E4M3], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38, 1e-30, 0.0], ids=str)
def test_append_of_values_no_scale_fits(codes, value):
    grow = torch.ones(9, 1)
    grow[4] = value
    check_append(Batch8([9], [9], 1, 1, 64, 8, codes, F32), 0, False, False, grow=grow)
    check_append(Batch8([9], [20], 1, 1, 64, 8, codes, F32), 0, False, False, grow=grow)
    check_append(Batch8([9], [9], 1, 1, 64, 16, codes, F32), 0, False, False, grow=torch.full((9, 1), value))


def test_a_page_stays_nan_until_it_starts_afresh():
    b = Batch8([1], [1], 1, 1, 64, 8, I8, F32)
    pool, scales, batch = setup(b)
    x = torch.ones(1, 1, 64, device="cuda")
    page = int(b.page_table[0, 0])

    def step(length, value):
        batch._keep[1].fill_(length)
        batch.append(0, x, x * value, x)
        return float(scales[page, 0, 0, 0])

    import math
    assert step(1, 1.0) == pytest.approx(1 / 127)
    assert math.isnan(step(2, float("inf"))) and math.isnan(step(3, 1.0))
    assert step(1, 2.0) == pytest.approx(2 / 127)
    assert float(scales[page, 0, 1, 0]) == pytest.approx(1 / 127)


def test_one_token_at_a_time_gives_a_page_the_scale_of_its_largest():
    """A page filled by 16 calls: the scale is what one call would choose, the codes are off by the roundings of its growths."""
    b = Batch8([16], [16], 2, 2, 64, 16, I8, F32)
    x = torch.randn(16, 2, 64, generator=torch.Generator().manual_seed(1)).cuda()
    pool, scales, whole = setup(b)
    whole.append(0, x, x, x)
    one = Batch8([1], [16], 2, 2, 64, 16, I8, F32)
    pool1, scales1, step = setup(one)
    grown = torch.zeros(2, 2)
    for i in range(16):
        step._keep[1].fill_(i + 1)
        before = scales1[int(one.page_table[0, 0]), 0].clone()
        step.append(0, x[i:i + 1], x[i:i + 1], x[i:i + 1])
        grown += (scales1[int(one.page_table[0, 0]), 0] != before).cpu() * (i > 0)
    at, at1 = int(b.page_table[0, 0]), int(one.page_table[0, 0])
    assert torch.equal(scales[at, 0], scales1[at1, 0])
    off = (pool[at, 0].int() - pool1[at1, 0].int()).abs().cpu()
    assert (off <= 0.5 * grown[..., None, None] + 1).all()             # half a step per growth (all later scales are larger), and the final rounding


def test_append_in_place_and_unaligned_rows():
    b = Batch8([7, 6], [7, 30], 4, 4, 64, 16, I8)
    table = rows_of(b, 64, False)[3].cuda()
    pool, scales, batch = setup(b)
    x = torch.randn(13, 3, 4, 64, device="cuda").to(BF16)
    q, k, v = (x[:, j].contiguous() for j in range(3))
    ref = batch.append(0, q, k, v, rope=table)
    pool_ref, scales_ref = pool.clone(), scales.clone()
    odd = torch.zeros(13, 3 * 256 + 1, device="cuda", dtype=BF16)                   # rows that start on odd elements
    odd[:, 1:] = x.reshape(13, -1)
    qo, ko, vo = (odd[:, 1 + 256 * j:257 + 256 * j].view(13, 4, 64) for j in range(3))
    pool.copy_(b.pool.cuda())
    scales.copy_(b.scales.cuda())
    got = batch.append(0, qo, ko, vo, rope=table)
    same = lambda a, c: ((a == c) | (a.isnan() & c.isnan())).all()
    assert torch.equal(got, ref) and torch.equal(pool, pool_ref) and same(scales, scales_ref)
    assert batch.append(0, q, k, v, rope=table, out=q).data_ptr() == q.data_ptr()
    assert torch.equal(q, ref)


# ----------------------------------------------------------------------------------------------- attention
ATTENTION = [
    # rows, cached, heads, kv heads, dim, page, codes, type, prefix
    ([1], [1], 1, 1, 64, 16, I8, BF16, 0),
    ([1, 1], [60, 9], 4, 4, 64, 16, I8, BF16, 100),
    ([1] * 5, [1, 64, 65, 200, 513], 8, 2, 128, 16, I8, BF16, 0),
    ([1] * 5, [1, 64, 65, 200, 513], 8, 2, 128, 16, E4M3, F16, 333),
    ([9] * 3, [9, 100, 1030], 14, 2, 128, 32, E4M3, F16, 301),
    ([3, 0, 16, 1], [10, 5, 16, 0], 16, 2, 128, 8, I8, BF16, 17),     # an empty sequence; a row with nothing of its own
    ([2, 4], [1, 0], 4, 2, 128, 16, I8, BF16, 0),                     # rows that see nothing
    ([128], [128], 2, 2, 128, 16, I8, BF16, 0),
    ([127, 129, 1, 300], [127, 129, 1, 300], 4, 1, 128, 16, E4M3, BF16, 0),
    ([257, 31], [400, 700], 8, 8, 64, 64, I8, F16, 0),
    ([32] * 6, [32] * 6, 5, 5, 128, 16, I8, BF16, 200),               # scoring windows
    ([20, 44], [20, 90], 8, 1, 128, 128, E4M3, F16, 129),
    ([40, 7], [333, 60], 6, 3, 80, 16, I8, BF16, 70),
    ([40, 7], [333, 60], 9, 3, 96, 32, E4M3, F16, 0),
    ([3, 1], [90, 40], 4, 2, 16, 8, I8, BF16, 33),
    ([3, 70], [90, 140], 4, 2, 48, 64, E4M3, BF16, 33),
    ([4, 70], [90, 140], 8, 8, 128, 128, I8, BF16, 0),
    ([5, 30], [33, 30], 4, 2, 128, 16, I8, F32, 40),                  # fp32 arithmetic: types, dims and groups the tensor cores do not take
    ([5, 30], [33, 30], 4, 2, 40, 16, E4M3, BF16, 40),
    ([5, 30], [33, 30], 4, 2, 50, 16, I8, F16, 0),
    ([5, 30], [33, 30], 2, 1, 256, 32, I8, BF16, 0),
    ([5, 3], [33, 300], 260, 2, 64, 32, I8, BF16, 0),
]


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c[2:]))
def test_attention(case, form):
    n, kv, H, Hk, D, page, codes, xt, prefix = case
    b = Batch8(n, kv, H, Hk, D, page, codes, xt, blocks=2, block=1, prefix_len=prefix, padding=2, spread=3.0)
    pool, scales, batch = setup(b)
    out = torch.full((b.n_rows, H, D), 3.0, device="cuda", dtype=xt)
    got = (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(1, b.q.cuda(), out=out)
    assert got.data_ptr() == out.data_ptr()
    want, tol = attention8(b, b.pool, b.scales, b.q)
    want[b.start[-1]:] = 3.0                                             # padding rows keep what out held
    close(out, want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("codes", [I8, E4M3], ids=str)
def test_far_scores_unlike_scales_and_strided_queries(codes, form):
    """Scores in the hundreds, scales that differ by up to 2^40 from page to page, queries sliced out of a wider tensor."""
    b = Batch8([40, 1], [300, 77], 8, 2, 128, 16, codes, BF16, spread=20.0)
    b.scales[:, :, 0] = 1 / 40.0
    pool, scales, batch = setup(b)
    wide = torch.zeros(b.n_rows, 12, 128, dtype=BF16)
    wide[:, 2:10] = b.q * 8
    q = wide.cuda()[:, 2:10]
    want, tol = attention8(b, b.pool, b.scales, wide[:, 2:10])
    close((batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, q), want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_scores_of_thousands(form):
    b = Batch8([40, 1], [300, 77], 4, 4, 64, 32, I8, BF16, spread=2.0)
    b.q *= 2000
    pool, scales, batch = setup(b)
    want, tol = attention8(b, b.pool, b.scales, b.q)
    close((batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, b.q.cuda()), want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("xt", [BF16, F16, F32], ids=str)
def test_rows_that_see_a_nan_scale_are_nan_and_no_others(xt, form):
    b = Batch8([30, 5], [30, 40], 4, 2, 64, 8, I8, xt)
    b.scales[int(b.page_table[0, 2]), 0, 0, 1] = float("nan")              # positions 16..23 of the first sequence, kv head 1, K
    pool, scales, batch = setup(b)
    out = (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, b.q.cuda()).cpu()
    assert out[16:30, 2:].isnan().all()
    clean = Batch8([30, 5], [30, 40], 4, 2, 64, 8, I8, xt)
    want, tol = attention8(clean, clean.pool, clean.scales, clean.q)
    keep = torch.ones(35, 4, dtype=torch.bool)
    keep[16:30, 2:] = False
    if xt == F32:
        keep[:16, 2:] = False                                            # fp32 arithmetic: a later row's NaN may reach rows of its sequence
    close(out[keep], want[keep], tol[keep])


def test_empty_pages_with_scale_zero():
    b = Batch8([3], [40], 2, 2, 64, 8, I8)
    for pg in (int(b.page_table[0, 0]), int(b.page_table[0, 3])):
        b.scales[pg, 0] = 0.0
        b.pool[pg, 0] = 0
    pool, scales, batch = setup(b)
    want, tol = attention8(b, b.pool, b.scales, b.q)
    close(batch.prefix_attention(0, b.q.cuda()), want, tol)
    close(batch.prompt_attention(0, b.q.cuda()), want, tol)
    b.scales[:], b.pool[:] = 0.0, 0
    pool.copy_(b.pool), scales.copy_(b.scales)
    assert (batch.prefix_attention(0, b.q.cuda()) == 0).all() and (batch.prompt_attention(0, b.q.cuda()) == 0).all()


def test_append_then_attention_then_a_token():
    """A decoding step as a program runs it: 8-bit append, attention over what it wrote, a projection, a token."""
    from paper_2410_06916_b200 import sample_rows
    b = Batch8([1] * 6, [5, 17, 1, 64, 33, 90], 8, 2, 64, 16, I8, BF16)
    pool, scales, batch = setup(b)
    x, cut, _, table = rows_of(b, 64, False)
    q, k, v = cut(x.cuda())
    q = batch.append(0, q, k, v, rope=table.cuda())
    o = batch.prefix_attention(0, q)
    codes, sc, _ = append8(b, b.pool, b.scales, *cut(x)[1:], table)
    want, tol = attention8(b, as_codes(codes, I8), sc, q.cpu())
    close(o, want, tol)
    w = torch.randn(512, 1000, generator=torch.Generator().manual_seed(2)).cuda()
    logits = o.float().view(6, 512) @ w
    tokens, probs = sample_rows(logits, torch.full((6,), 0.5, device="cuda"), temperature=0.0)
    assert torch.equal(tokens.long(), logits.argmax(1)) and (probs == 1).all()


# ----------------------------------------------------------------------------------------------- how the calls are used
def run(batch, form, q, **kw):
    return (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, q, **kw)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("rows,cached,heads,kv_heads", [(1, 40, 8, 2), (20, 0, 8, 1), (70, 300, 4, 4), (9, 500, 14, 2)])
def test_many_short_sequences_give_the_same_bits_every_time(form, rows, cached, heads, kv_heads):
    """Pieces of one or a few key tiles, many per SM: what one role of the many-row kernel does runs ahead of another's."""
    n = [rows + i % 3 for i in range(200)]
    b = Batch8(n, [x + (i * 37) % (cached + 1) for i, x in enumerate(n)], heads, kv_heads, 64, 16, I8)
    pool, scales, batch = setup(b)
    q = b.q.cuda()
    want, tol = attention8(b, b.pool, b.scales, b.q, dev="cuda")
    first = run(batch, form, q)
    close(first, want, tol)
    for _ in range(20):
        assert torch.equal(run(batch, form, q), first)


@pytest.mark.parametrize("codes", [I8, E4M3], ids=str)
def test_pools_beyond_2_to_the_32_bytes(codes):
    """Pages at the end of a pool of 5 GB."""
    from paper_2410_06916_b200 import PagedKV, RowBatch
    b = Batch8([3, 40], [200, 300], 16, 8, 128, 128, codes, prefix_len=130)
    far = 20000
    pool = torch.zeros((far,) + b.pool.shape[1:], dtype=torch.uint8, device="cuda").view(codes)
    scales = torch.full((far,) + b.scales.shape[1:], float("nan"), device="cuda")
    shift = far - b.n_pages
    pool.view(torch.uint8)[shift:] = b.pool.view(torch.uint8).cuda()
    scales[shift:] = b.scales.cuda()
    args, kw = b.device_args()
    live = args[2] < b.n_pages
    args[2][live] += shift
    kw["prefix_pages"] += shift
    batch = RowBatch(PagedKV(pool, scales), *args, **kw)
    want, tol = attention8(b, b.pool, b.scales, b.q)
    for form in ("prompt", "prefix"):
        close(run(batch, form, b.q.cuda()), want, tol)
    b32 = Batch8([3, 40], [200, 300], 16, 8, 128, 128, codes, F32, prefix_len=130)
    want, tol = attention8(b32, b.pool, b.scales, b32.q)
    close(run(batch, "prompt", b32.q.cuda()), want, tol)
    x, cut, _, table = rows_of(b, 128, False)
    batch.append(0, *cut(x.cuda()), rope=table.cuda())
    code, sc, near = append8(b, b.pool, b.scales, *cut(x)[1:], table)
    got = pool[shift:].view(torch.uint8).view(codes).cpu().to(F64)
    assert ((got == code) | (got.isnan() & code.isnan()) | (near & ((got - code).abs() <= 1))).all()
    got = scales[shift:].cpu()
    assert ((got == sc) | (got.isnan() & sc.isnan())).all()


def test_four_thousand_sequences():
    n = [1] * 4096
    b = Batch8(n, [1 + i % 40 for i in range(4096)], 2, 1, 64, 8, I8)
    pool, scales, batch = setup(b)
    q = b.q.cuda()
    a, c = run(batch, "prompt", q), run(batch, "prefix", q)
    pick = [0, 1, 31, 32, 33, 1023, 2048, 4095]
    small = Batch8(n, b.kv, 2, 1, 64, 8, I8)
    small.n = [1 if i in pick else 0 for i in range(4096)]              # the definition, for a few of them
    want, tol = attention8(small, b.pool, b.scales, b.q)
    close(a[pick], want[pick], tol[pick])
    close(c[pick], want[pick], tol[pick])


def test_a_captured_step_follows_lengths_tables_and_values():
    b = Batch8([1] * 5, [30, 17, 64, 1, 100], 8, 2, 64, 16, I8)
    pool, scales, batch = setup(b)
    x, cut, _, table = rows_of(b, 64, False)
    table, xd = table.cuda(), x.cuda()

    def step():
        q = batch.append(0, *cut(xd), rope=table)
        return run(batch, "prefix", q), run(batch, "prompt", q)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):                                                   # two graphs, each with workspaces of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = step()
        graphs.append((g, outs))
    for seed, shorter in ((6, 0), (7, 12)):
        pool.copy_(b.pool), scales.copy_(b.scales)
        new = rows_of(b, 64, False, seed=seed)[0]
        xd.copy_(new)
        kv = [max(1, l - shorter) for l in b.kv]
        batch._keep[1].copy_(torch.tensor(kv, dtype=torch.int32))
        for g, outs in graphs:
            pool.copy_(b.pool), scales.copy_(b.scales)
            g.replay()
            moved = Batch8(b.n, b.kv, 8, 2, 64, 16, I8)
            moved.kv = kv
            code, sc, _ = append8(moved, b.pool, b.scales, *cut(new)[1:], table.cpu())
            q = torch.empty_like(moved.q)
            batch2 = setup(b)[2]
            batch2._keep[1].copy_(torch.tensor(kv, dtype=torch.int32))
            q = batch2.append(0, *cut(new.cuda()), rope=table).cpu()
            want, tol = attention8(moved, as_codes(code.nan_to_num(0.0), I8), sc, q)
            for o in outs:
                close(o, want, tol)


def test_a_given_stream_and_inputs_that_are_freed():
    b = Batch8([3, 40], [200, 90], 8, 2, 128, 32, E4M3, F16)
    pool, scales, batch = setup(b)
    want = [run(batch, form, b.q.cuda()) for form in ("prompt", "prefix")]
    side = torch.cuda.Stream()
    for form, w in zip(("prompt", "prefix"), want):
        q = b.q.cuda()
        side.wait_stream(torch.cuda.current_stream())
        got = run(batch, form, q, stream=side)
        del q
        junk = torch.full((b.n_rows, 8, 128), 7.0, dtype=F16, device="cuda")   # (memory of q, were it handed out)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, w) and (junk == 7).all()


WAITS = [
    # rows of each of four sequences, cached, heads, kv heads, dim, codes, type, prefix, form
    (40, 300, 8, 2, 128, I8, BF16, 0, "prompt"),
    (1, 300, 8, 2, 64, E4M3, F16, 100, "prefix"),                # the few-row kernel, 8 rows, and the prefix with it
    (9, 900, 14, 2, 128, I8, F16, 2000, "prefix"),               # ... 64 rows, beside the many-row kernel
    (40, 100, 8, 1, 128, I8, BF16, 20000, "prefix"),             # the many-row kernel alone
]


def waits_run_out(case):
    """In a process of its own: the probe gives up, the report comes once, the next call on the same workspace is right."""
    import ctypes as C
    from paper_2410_06916_b200 import SwiftError, batch_sync, lib
    from paper_2410_06916_b200.binding import _DevBuf
    each, kv, H, Hk, dim, codes, xt, prefix, form = WAITS[case]
    b = Batch8([each] * 4, [kv, kv - 9, kv // 2, kv], H, Hk, dim, 16, codes, xt, prefix_len=prefix)
    pool, scales, batch = setup(b)
    want, tol = attention8(b, b.pool, b.scales, b.q, dev="cuda")
    q = b.q.cuda()
    rows, x = 0 if form == "prompt" else batch.max_rows, {BF16: 1, F16: 2}[xt]
    need = lib().swift_coded_prefix_workspace_bytes(batch._kv_p, batch._c_p, H, max(rows, 1), x)
    out = torch.empty_like(q)
    a = batch._attention(0, q, None)
    a.out = out.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    for fill in (0, 0x7F, 0xFF, 0x01):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")       # what an entry no one wrote may hold
        where = _DevBuf(ws.data_ptr(), need)
        assert lib().swift_probe_coded_wait_limit(batch._kv_p, batch._c_p, C.byref(a), x, rows, where, 1000, stream) == 0
        try:
            batch_sync()
            raise AssertionError("no report")
        except SwiftError as e:
            assert "ETIMEOUT" in str(e), e
        batch_sync()
        if form == "prefix":
            assert lib().swift_coded_prefix_attention(batch._kv_p, batch._c_p, C.byref(a), x, rows, where, stream) == 0
        else:
            assert lib().swift_coded_prompt_attention(batch._kv_p, batch._c_p, C.byref(a), x, stream) == 0
        batch_sync()
        close(out, want, tol)
    assert lib().swift_probe_coded_wait_limit(batch._kv_p, batch._c_p, C.byref(a), 0, rows, where, 1000, stream) == 6


@pytest.mark.parametrize("case", range(len(WAITS)))
def test_a_wait_that_runs_out_is_a_status(case):
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    code = (f"import sys; sys.path[:0] = [{here!r}, {os.path.dirname(here)!r}]\nimport torch\nimport test_paged8_gpu as t\n"
            f"t.waits_run_out({case})\ntorch.cuda.synchronize()\nprint('fine')\n")
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "fine" in done.stdout, done.stderr[-2000:]


def test_refusals_of_the_python_side():
    from paper_2410_06916_b200 import PagedKV, sample_rows
    pool = torch.zeros(4, 1, 2, 2, 16, 64, dtype=torch.int8, device="cuda")
    scales = torch.zeros(4, 1, 2, 2, device="cuda")
    for p, s in ((pool, scales[:3]), (pool, scales.half()), (pool.to(BF16), scales), (pool, None), (pool, scales.cpu()), (pool.transpose(3, 4), scales),
                 (pool, scales.clone().requires_grad_())):
        with pytest.raises(ValueError):
            PagedKV(p, s)
    b = Batch8([2], [5], 4, 2, 64, 16, I8)
    _, _, batch = setup(b)
    with pytest.raises(TypeError):
        batch.prompt_attention(0, b.q.cuda().double())
    with pytest.raises(TypeError):
        batch.append(0, b.q.cuda(), b.q.cuda()[:, :2].float(), b.q.cuda()[:, :2])
    with pytest.raises(ValueError):
        batch.prefix_attention(0, b.q.cuda(), out=torch.empty(2, 4, 64, device="cuda"))
    with pytest.raises(ValueError):
        batch.prefix_attention(0, b.q.cuda().requires_grad_())
    x, u = torch.zeros(2, 10, device="cuda"), torch.zeros(2, device="cuda")
    for bad in (dict(uniforms=u[:1]), dict(uniforms=u.double()), dict(temperature=-1.0), dict(temperature=float("nan")), dict(top_p=float("nan")),
                dict(min_p=1.5), dict(top_k=1 << 40), dict(top_k=torch.zeros(2, device="cuda")), dict(tokens=torch.zeros(2, device="cuda")),
                dict(logits=x.t()), dict(logits=x.double()), dict(logits=x.clone().requires_grad_()), dict(logits=x[0])):
        with pytest.raises(ValueError):
            sample_rows(**{"logits": x, "uniforms": u, **bad})
    from paper_2410_06916_b200 import SwiftError
    with pytest.raises(SwiftError):
        sample_rows(torch.zeros(1, 262145, device="cuda"), u[:1])
