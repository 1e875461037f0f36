"""The paged-batch operators on the GPU against their 64-bit definitions (tests/paged_reference.py derives the bounds)."""
import pytest
import torch

from paged_reference import (F64, Batch, append_tolerance, attention, finish_heads, frequencies, half_step, table)

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def setup(b: Batch, **more):
    from paper_2410_06916_b200 import PagedKV, RowBatch
    args, kw = b.device_args()
    kw.update(more)
    pool = b.pool.cuda()
    return pool, RowBatch(PagedKV(pool), *args, **kw)


def close(got, want, tol):
    got = got.to(F64).cpu()
    want, tol = want.cpu(), tol.cpu()
    assert torch.isfinite(got).all()
    off = (got - want).abs() - tol
    assert (off <= 0).all(), f"{int((off > 0).sum())} of {off.numel()} outside; worst {float(off.max())} over, at {(off == off.max()).nonzero()[0].tolist()}"


# ----------------------------------------------------------------------------------------------- rope
@pytest.mark.parametrize("kw", [dict(n=1, R=2), dict(n=33, R=64), dict(n=4096, R=128), dict(n=777, R=80, theta=5e5, factor=8.0),
                                dict(n=70001, R=128, theta=5e5, factor=8.0, original=8192, low=1.0, high=4.0),
                                dict(n=2000, R=96, theta=1e4, factor=32.0, original=2048, low=1.0, high=32.0, magnitude=1.3466)], ids=str)
def test_rope_table(kw):
    from paper_2410_06916_b200 import rope_table
    kw = dict(kw)
    n, R, mag = kw.pop("n"), kw.pop("R"), kw.pop("magnitude", 1.0)
    names = {"original": "original_positions", "low": "low_turns", "high": "high_turns"}
    got = rope_table(n, R, magnitude=mag, **{names.get(k, k): v for k, v in kw.items()})
    want = table(n, R, magnitude=mag, **kw)
    # one rounding to fp32, and angles good to a few steps of 2^-53 of the position (both sides)
    close(got, want, 2.0 ** -24 * want.abs() + mag * n * 2.0 ** -49)


def test_rope_table_writes_no_further_than_its_end():
    from paper_2410_06916_b200 import rope_table
    buf = torch.full((100, 32, 2), 7.0, device="cuda")
    rope_table(37, 64, out=buf[:37])
    assert (buf[37:] == 7).all() and (buf[:37].abs() <= 1).all()
    assert rope_table(0, 64).shape == (0, 32, 2)


# ----------------------------------------------------------------------------------------------- append
def check_append(b: Batch, x_dtype, R, interleaved, norm, positions=None, strided=True, eps=1e-5):
    from paper_2410_06916_b200 import rope_table
    pool, batch = setup(b)
    H, Hk, D, T = b.heads, b.kv_heads, b.dim, b.n_rows
    g = torch.Generator().manual_seed(5)
    width = (H + 2 * Hk) * D + (16 if strided else 0)
    x = torch.randn(T, width, generator=g).to(x_dtype)
    q, k, v = x[:, :H * D].view(T, H, D), x[:, H * D:(H + Hk) * D].view(T, Hk, D), x[:, (H + Hk) * D:(H + 2 * Hk) * D].view(T, Hk, D)
    gains = (1 + 0.2 * torch.randn(2, D, generator=g)) if norm else None
    xd = x.cuda()
    qd, kd, vd = xd[:, :H * D].view(T, H, D), xd[:, H * D:(H + Hk) * D].view(T, Hk, D), xd[:, (H + Hk) * D:(H + 2 * Hk) * D].view(T, Hk, D)
    longest = b.prefix_len + max(b.kv + [0]) + 1
    rope = rope_table(longest, R) if R else None
    before = pool.clone()
    out = torch.full((T, H, D), 3.0, device="cuda", dtype=b.dtype)
    gd = gains.cuda() if norm else None
    got = batch.append(b.block, qd, kd, vd, rope=rope, interleaved=interleaved, q_gain=gd[0] if norm else None,
                       k_gain=gd[1] if norm else None, eps=eps, positions=None if positions is None else positions.cuda(), out=out)
    assert got.data_ptr() == out.data_ptr()
    freq = frequencies(R) if R else None
    want_pool, tol_pool = before.cpu().to(F64), torch.zeros(before.shape, dtype=F64)
    want_q, tol_q = torch.full((T, H, D), 3.0, dtype=F64), torch.zeros(T, H, D, dtype=F64)
    for i, n in enumerate(b.n):
        own = torch.arange(n) + b.kv[i] - n
        rows = torch.arange(b.start[i], b.start[i] + n)
        keep = own >= 0
        own, rows = own[keep], rows[keep]
        pages = b.page_table[i].long()[own // b.page] if len(own) else own
        keep = (pages >= 0) & (pages < b.n_pages)
        pos = own + b.prefix_len if positions is None else positions[rows].long()
        if R:
            keep &= (pos >= 0) & (pos < longest)
        own, rows, pages, pos = own[keep], rows[keep], pages[keep], pos[keep]
        if len(rows) == 0:
            continue
        yq, mq = finish_heads(q[rows], pos, freq, interleaved, gains[0] if norm else None, eps)
        yk, mk = finish_heads(k[rows], pos, freq, interleaved, gains[1] if norm else None, eps)
        want_q[rows], tol_q[rows] = yq, append_tolerance(yq, mq, D, b.dtype)
        for j in range(len(rows)):
            want_pool[pages[j], b.block, 0, :, own[j] % b.page] = yk[j]
            tol_pool[pages[j], b.block, 0, :, own[j] % b.page] = append_tolerance(yk[j], mk[j], D, b.dtype)
            yv = v[rows[j]].to(F64)
            want_pool[pages[j], b.block, 1, :, own[j] % b.page] = yv
            tol_pool[pages[j], b.block, 1, :, own[j] % b.page] = half_step(b.dtype) * yv.abs() + (2.0 ** -25 if b.dtype == F16 else 0.0)
    close(out, want_q, tol_q)
    got_pool = pool.cpu().to(F64)
    both = torch.isnan(want_pool) & torch.isnan(got_pool)              # slots nothing was written to keep their NaN
    close(torch.where(both, torch.zeros_like(got_pool), got_pool), torch.where(both, torch.zeros_like(want_pool), want_pool), tol_pool)


APPEND = [
    # n rows, cached, heads, kv heads, dim, page, cache type, x type, rotary dims, pairs side by side, norm
    ([1], [1], 4, 4, 64, 16, BF16, BF16, 64, False, False),
    ([5, 0, 1, 40], [5, 7, 33, 45], 8, 2, 128, 16, BF16, BF16, 128, False, True),
    ([3, 17], [20, 17], 7, 1, 128, 8, F16, F32, 128, True, True),
    ([9] * 33, [9 + i for i in range(33)], 4, 2, 64, 32, BF16, F32, 32, False, False),
    ([2] * 70, [2 + 3 * i for i in range(70)], 2, 2, 16, 8, F32, F32, 16, False, True),
    ([13, 4], [13, 4], 3, 3, 80, 64, F16, F16, 32, True, True),
    ([13, 4], [13, 4], 3, 3, 80, 64, BF16, BF16, 80, False, True),
    ([6, 2], [6, 9], 2, 1, 256, 128, BF16, BF16, 128, False, True),
    ([6, 2], [6, 9], 4, 2, 96, 16, BF16, F32, 0, False, True),        # no rotation
    ([6, 2], [6, 9], 5, 5, 34, 16, F32, F32, 10, False, True),        # dims and rotated dims of no particular size
    ([6, 2], [6, 9], 5, 1, 50, 16, F16, F16, 50, True, False),
    ([4, 3], [2, 1], 2, 2, 64, 16, BF16, BF16, 64, False, False),     # more rows than cached positions: the first are left out
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c[2:]))
def test_append(case):
    n, kv, H, Hk, D, page, dt, xt, R, inter, norm = case
    check_append(Batch(n, kv, H, Hk, D, page, dt, padding=3, blocks=2, block=1, poison=True), xt, R, inter, norm)


def test_append_behind_a_prefix_and_at_given_positions():
    b = Batch([4, 2, 5], [11, 2, 70], 4, 2, 128, 16, BF16, prefix_len=21)
    check_append(b, BF16, 128, False, True)
    depth = torch.tensor([7, 8, 8, 9, 21, 22, 0, 1000000, -1, 60, 61], dtype=torch.int32)   # two of them outside the table
    check_append(b, BF16, 128, False, False, positions=depth)


def test_append_leaves_out_rows_whose_page_is_outside_the_pool():
    b = Batch([4, 20], [20, 20], 4, 2, 64, 8, BF16, blocks=2)
    b.page_table[1, 1] = -5
    b.page_table[1, 2] = b.n_pages
    b.page_table[0, 2] = 1 << 30
    check_append(b, BF16, 64, False, True)


def test_append_in_place_and_unaligned_rows():
    from paper_2410_06916_b200 import rope_table
    b = Batch([7, 6], [7, 30], 4, 4, 64, 16, BF16, poison=False)
    pool, batch = setup(b)
    x = torch.randn(13, 3, 4, 64, device="cuda").to(BF16)
    rope = rope_table(64, 64)
    q, k, v = (x[:, j].contiguous() for j in range(3))
    ref = batch.append(0, q, k, v, rope=rope)
    pool_ref = pool.clone()
    odd = torch.zeros(13, 3 * 256 + 1, device="cuda", dtype=BF16)                   # rows that start on odd elements
    odd[:, 1:] = x.reshape(13, -1)
    qo, ko, vo = (odd[:, 1 + 256 * j:257 + 256 * j].view(13, 4, 64) for j in range(3))
    pool.zero_()
    pool.copy_(b.pool.cuda())
    got = batch.append(0, qo, ko, vo, rope=rope)
    assert torch.equal(got, ref) and torch.equal(pool, pool_ref)
    assert batch.append(0, q, k, v, rope=rope, out=q).data_ptr() == q.data_ptr()
    assert torch.equal(q, ref)


# ----------------------------------------------------------------------------------------------- attention
ATTENTION = [
    # rows, cached, heads, kv heads, dim, page, type, prefix
    ([1], [1], 1, 1, 64, 16, BF16, 0),
    ([1, 1], [60, 9], 4, 4, 64, 16, BF16, 100),
    ([1] * 5, [1, 64, 65, 200, 513], 8, 2, 128, 16, BF16, 0),
    ([1] * 5, [1, 64, 65, 200, 513], 8, 2, 128, 16, F16, 333),
    ([9] * 3, [9, 100, 1030], 14, 2, 128, 32, F16, 301),
    ([3, 0, 16, 1], [10, 5, 16, 0], 16, 2, 128, 8, BF16, 17),       # an empty sequence; a row with nothing of its own
    ([2, 4], [1, 0], 4, 2, 128, 16, BF16, 0),                       # rows that see nothing
    ([128], [128], 2, 2, 128, 16, BF16, 0),
    ([127, 129, 1, 300], [127, 129, 1, 300], 4, 1, 128, 16, BF16, 0),
    ([257, 31], [400, 700], 8, 8, 64, 64, F16, 0),
    ([32] * 6, [32] * 6, 5, 5, 128, 16, BF16, 200),                 # scoring windows
    ([20, 44], [20, 90], 8, 1, 128, 128, F16, 129),
    ([40, 7], [333, 60], 6, 3, 80, 16, BF16, 70),
    ([40, 7], [333, 60], 9, 3, 96, 32, F16, 0),
    ([5, 1], [50, 61], 4, 4, 16, 16, BF16, 40),
    ([5, 70], [50, 161], 12, 1, 8, 16, F16, 40),
    ([33, 2], [50, 200], 7, 1, 120, 8, BF16, 0),
    ([3, 50], [90, 61], 4, 2, 128, 16, F32, 40),
    ([3, 50], [90, 61], 4, 2, 256, 16, BF16, 40),
    ([3, 20], [90, 61], 4, 2, 36, 16, F16, 40),
    ([16, 16], [700, 20], 64, 8, 128, 16, BF16, 1100),              # 128 packed rows per sequence and kv head
    ([700], [700], 3, 1, 128, 32, F16, 0),
    ([2] * 150, [2 + 5 * i for i in range(150)], 4, 2, 64, 16, BF16, 77),
]
IDS = lambda c: "-".join(str(x).replace("torch.", "") for x in [len(c[0]), max(c[0]), max(c[1])] + list(c[2:]))


@pytest.mark.parametrize("case", ATTENTION, ids=IDS)
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_attention(case, form):
    n, kv, H, Hk, D, page, dt, prefix = case
    b = Batch(n, kv, H, Hk, D, page, dt, prefix_len=prefix, padding=2, blocks=2, block=1)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    out = torch.full((b.n_rows, H, D), 5.0, device="cuda", dtype=dt)
    q = b.q.cuda()
    q[b.start[-1]:] = float("nan")                                   # padding rows are not read
    (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(1, q, out=out)
    assert (out[b.start[-1]:] == 5).all()                            # ... nor written
    close(out[:b.start[-1]], want[:b.start[-1]], tol[:b.start[-1]])
    again = (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(1, q)
    assert torch.equal(again[:b.start[-1]], out[:b.start[-1]])       # the same bits, whatever order the blocks ran in


@pytest.mark.parametrize("case", [
    ([5, 9, 1], [2, 0, 30], 4, 2, 128, 16, BF16, 100),              # the few-row kernel beside the many-row kernel
    ([5, 2], [2, 0], 2, 2, 64, 16, F16, 70),                        # the few-row kernel alone
    ([70, 33], [60, 2], 8, 2, 128, 32, BF16, 300),                  # the many-row kernel
    ([5, 9], [2, 0], 4, 2, 36, 16, F32, 40),
], ids=IDS)
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_rows_before_their_sequences_first_position_see_the_prefix(case, form):
    test_attention(case, form)


# enough rows for blocks of 64 in fp32 arithmetic: at least 148 of them
FP32_MANY = [
    ([300, 0, 40], [300, 7, 333], 32, 8, 128, 16, F32, 0),
    ([700, 1, 650], [700, 90, 1000], 8, 8, 36, 16, F32, 40),
    ([1300, 60], [1300, 61], 8, 8, 66, 8, BF16, 0),                 # 4-byte rows: elements are staged one by one
    ([640, 30], [650, 25], 16, 8, 256, 32, F16, 33),                # two chunks of dims; rows with nothing of their own
    ([1300, 50], [1290, 70], 8, 8, 130, 64, F32, 0),                # rows that see nothing; an odd second chunk
]


@pytest.mark.parametrize("case", FP32_MANY, ids=IDS)
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_attention_in_fp32_arithmetic_with_many_rows(case, form):
    test_attention(case, form)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_fp32_arithmetic_with_many_rows_leaves_out_rows_and_pages(form):
    """Pages outside the pool, a sequence of NaN, rows beyond max_rows: 700 rows of 8 heads each, in fp32."""
    b = Batch([700, 650], [700, 800], 8, 8, 64, 16, F32, prefix_len=90)
    q = b.q.clone()
    q[:700] = float("nan")
    b.page_table[1, 3] = b.n_pages
    b.page_table[1, 20] = -1
    pool, batch = setup(b, max_rows=640)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    out = torch.full((b.n_rows, 8, 64), 5.0, device="cuda", dtype=F32)
    (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, q.cuda(), out=out)
    kept = 650 if form == "prompt" else 640
    close(out[700:700 + kept], want[700:700 + kept], tol[700:700 + kept])
    assert (out[700 + kept:] == 5).all()
    assert torch.isnan(out[:640]).all()


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("heads,kv_heads,each", [(14, 2, 9), (14, 2, 1), (56, 8, 40), (9, 3, 40)])
def test_bits_do_not_depend_on_what_ran_before(form, heads, kv_heads, each):
    """Groups that leave rows of a tile unused: what an earlier call left in shared memory for those rows must not show."""
    b = Batch([each] * 5, [300 + each] * 5, heads, kv_heads, 128, 16, BF16, prefix_len=500)
    pool, batch = setup(b)
    q = b.q.cuda()
    before = []
    for scale in (1.0, 1e3, 1e-3, 30.0):
        other = Batch([64, 33], [400, 90], 8, 1, 128, 16, BF16, prefix_len=70, seed=7)   # fills whole tiles
        opool, obatch = setup(other)
        (obatch.prompt_attention if form == "prompt" else obatch.prefix_attention)(0, other.q.cuda() * scale)
        before.append((batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, q))
    for o in before[1:]:
        assert torch.equal(o, before[0])


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("dim,dt", [(128, BF16), (64, F16), (128, F32)])
def test_attention_with_strided_queries_and_a_scale(form, dim, dt):
    b = Batch([37, 3], [50, 400], 8, 2, dim, 16, dt, prefix_len=50)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, scale=0.31, dev="cuda")
    call = batch.prompt_attention if form == "prompt" else batch.prefix_attention
    fused = torch.full((40, 12, dim), float("nan"), device="cuda", dtype=dt)
    fused[:, 2:10] = b.q.cuda()
    close(call(0, fused[:, 2:10], scale=0.31), want, tol)
    swapped = b.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)         # [heads][rows][dim] in memory
    close(call(0, swapped, scale=0.31), want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("dim,dt,each", [(128, BF16, 1), (128, BF16, 40), (64, F16, 9), (128, F32, 3)])
def test_attention_over_bad_pages(form, dim, dt, each):
    """Positions on pages outside the pool hold nothing, in the prefix and in a sequence's own part; a sequence all of
    whose pages are outside sees the prefix only, one without a prefix sees nothing."""
    for prefix in (90, 0):
        b = Batch([each] * 4, [200, 150, 60, 300], 8, 2, dim, 16, dt, prefix_len=prefix)
        if prefix:
            b.prefix_pages[2] = -1
            b.prefix_pages[5] = b.n_pages
        b.page_table[0, 1], b.page_table[0, 3], b.page_table[0, 12] = 1 << 30, -(1 << 31), b.n_pages
        b.page_table[2, :] = -7
        pool, batch = setup(b)
        want, tol = attention(b, b.pool, b.q, dev="cuda")
        call = batch.prompt_attention if form == "prompt" else batch.prefix_attention
        close(call(0, b.q.cuda()), want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("each", [1, 3, 48])
def test_one_sequences_nan_stays_its_own(form, each):
    b = Batch([each, each, each], [100, 130, 64 + each], 8, 2, 128, 16, BF16, prefix_len=0)
    for p in range(0, 130, 16):                                      # sequence 1: NaN and infinity all over its pages
        b.pool[int(b.page_table[1, p // 16]), 0, 1] = float("nan")
        b.pool[int(b.page_table[1, p // 16]), 0, 0] = float("inf")
    b.q[each:2 * each] = float("nan")
    pool, batch = setup(b)
    call = batch.prompt_attention if form == "prompt" else batch.prefix_attention
    got = call(0, b.q.cuda()).cpu()
    b.n = [each, 0, each]
    b.start = [0, each, 2 * each, 3 * each]
    clean = torch.nan_to_num(b.pool, nan=0.0, posinf=0.0)
    want, tol = attention(b, clean, torch.nan_to_num(b.q, nan=0.0), dev="cuda")
    rows = list(range(each)) + list(range(2 * each, 3 * each))
    close(got[rows], want[rows], tol[rows])


@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("dt", [BF16, F16])
def test_scores_far_apart(form, dt):
    """A running maximum that climbs by hundreds from tile to tile, and one that never moves again after the first: the
    rescaling of what was summed so far must not lose anything."""
    b = Batch([2, 64], [700, 700], 4, 2, 128, 16, dt, prefix_len=150)
    for i, up in ((0, True), (1, False)):
        for p in range(700):
            pg, sl = int(b.page_table[i, p // 16]), p % 16
            b.pool[pg, 0, 0, :, sl] = 0.0
            b.pool[pg, 0, 0, :, sl, 0] = (p if up else 700 - p) * 0.25
    b.q[:, :, 0] = 6.0
    pool, batch = setup(b)
    # heights are multiples of 1/4 up to 175 (exact in both types below 2^8) times 6 times the scale: scores up to 93
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    call = batch.prompt_attention if form == "prompt" else batch.prefix_attention
    close(call(0, b.q.cuda()), want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_rows_beyond_max_rows_and_odd_row_starts(form):
    """What a wrong plan can say without harm: more rows than max_rows, row starts outside the tensors, lengths outside the
    page table.  Nothing out of bounds is touched and well-formed sequences keep their results."""
    from paper_2410_06916_b200 import PagedKV, RowBatch
    b = Batch([4, 4], [40, 70], 8, 2, 128, 16, BF16)
    (start, kv, table), kw = b.device_args()
    pool = b.pool.cuda()
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    kw["max_rows"] = 2
    q = b.q.cuda()
    out = torch.full((8, 8, 128), 9.0, device="cuda", dtype=BF16)
    batch = RowBatch(PagedKV(pool), start, kv, table, **kw)
    if form == "prefix":
        batch.prefix_attention(0, q, out=out)
        close(out[[0, 1, 4, 5]], want[[0, 1, 4, 5]], tol[[0, 1, 4, 5]])
        assert (out[[2, 3, 6, 7]] == 9).all()
    kw["max_rows"] = 8
    bad = torch.tensor([0, 4, 1 << 30], dtype=torch.int32, device="cuda")
    RowBatch(PagedKV(pool), bad, torch.tensor([40, -3], dtype=torch.int32, device="cuda"), table, **kw)
    batch = RowBatch(PagedKV(pool), bad, torch.tensor([40, 1 << 30], dtype=torch.int32, device="cuda"), table, **kw)
    got = (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, q)
    close(got[:4], want[:4], tol[:4])
    backwards = torch.tensor([8, 4, -2], dtype=torch.int32, device="cuda")
    batch = RowBatch(PagedKV(pool), backwards, kv, table, **kw)
    (batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, q)
    batch.append(0, q, q[:, :2], q[:, :2])
    torch.cuda.synchronize()


def test_a_cache_beyond_32_bit_offsets():
    """Pages whose elements lie past 2^31 in the pool."""
    from paper_2410_06916_b200 import PagedKV, RowBatch, rope_table
    n_pages, blocks, Hk, page, D = 600, 16, 8, 128, 128
    pool = torch.empty(n_pages, blocks, 2, Hk, page, D, device="cuda", dtype=BF16)
    assert pool.numel() > (1 << 31)
    small = Batch([3, 140], [130, 140], 16, Hk, D, page, BF16)
    where = torch.tensor([598, 599, 597, 530, 599 - 1][:small.n_pages], dtype=torch.long)
    where = torch.tensor([599 - i for i in range(small.n_pages)])
    for i in range(small.n_pages):
        pool[int(where[i]), 15] = small.pool[i, 0].cuda()
    table_big = torch.where(small.page_table < small.n_pages, where[small.page_table.clamp(max=small.n_pages - 1).long()].to(torch.int32), small.page_table)
    (start, kv, _), kw = small.device_args()
    batch = RowBatch(PagedKV(pool), start, kv, table_big.cuda(), **kw)
    want, tol = attention(small, small.pool, small.q, dev="cuda")
    q = small.q.cuda()
    close(batch.prompt_attention(15, q), want, tol)
    close(batch.prefix_attention(15, q), want, tol)
    k = torch.randn(small.n_rows, Hk, D, device="cuda").to(BF16)
    batch.append(15, q, k, k)
    pos = 130 - 1
    assert torch.equal(pool[int(where[int(small.page_table[0, pos // page])]), 15, 0, :, pos % page], k[2])


@pytest.mark.parametrize("dim,dt", [(128, BF16), (128, F16), (64, BF16), (64, F16), (96, BF16)])
@pytest.mark.parametrize("n,kv,heads,kv_heads,prefix,parts", [
    ([2, 1, 2], [300, 40, 900], 8, 2, 0, True),             # own parts only
    ([1, 1], [300, 40], 8, 2, 500, True),                   # few rows: the prefix beside them in the same kernel
    ([3] * 12, [300] * 12, 8, 2, 900, True),                # the prefix by the many-row kernel, own parts by the few-row kernel
    ([7] * 5, [100, 7, 300, 64, 900], 16, 2, 2000, True),   # the same at 56 packed rows
    ([24, 40], [1500, 40], 8, 1, 20000, True),              # both by the many-row kernel
    ([200, 190], [200, 300], 8, 1, 130, False),             # each sequence by itself
], ids=["own", "few", "beside", "beside56", "many", "alone"])
def test_every_form_of_the_prefix_call(dim, dt, n, kv, heads, kv_heads, prefix, parts):
    """The forms a batch's sizes can select; those that leave parts to be joined need a workspace that holds them."""
    import ctypes
    b = Batch(n, kv, heads, kv_heads, dim, 32, dt, prefix_len=prefix, padding=1)
    pool, batch = setup(b)
    need = batch._lib.swift_prefix_workspace_bytes(ctypes.byref(batch.kv._c), ctypes.byref(batch._c), heads, batch.max_rows)
    assert (need > 4096) == parts, need
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    close(batch.prefix_attention(0, b.q.cuda())[:b.start[-1]], want[:b.start[-1]], tol[:b.start[-1]])


@pytest.mark.parametrize("heads,kv_heads", [(128, 1), (65, 1), (160, 1), (100, 2)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_large_groups(heads, kv_heads, dt):
    b = Batch([5, 2], [70, 200], heads, kv_heads, 64, 16, dt, prefix_len=40)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    close(batch.prompt_attention(0, b.q.cuda()), want, tol)
    close(batch.prefix_attention(0, b.q.cuda()), want, tol)


def test_as_many_sequences_as_a_batch_takes():
    n = 4096
    b = Batch([1 if i % 3 else 0 for i in range(n)], [1 + i % 40 for i in range(n)], 4, 2, 64, 8, BF16, prefix_len=9, poison=False)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    close(batch.prompt_attention(0, b.q.cuda()), want, tol)
    close(batch.prefix_attention(0, b.q.cuda()), want, tol)


@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_broadcast_queries(form):
    """Strides of zero: one head's or one row's queries for all."""
    for pick in (lambda q: q[:, :1], lambda q: q[:1]):
        b = Batch([40, 3], [50, 60], 8, 2, 128, 16, BF16, prefix_len=30)
        one = pick(b.q).clone()
        b.q[:] = one
        pool, batch = setup(b)
        want, tol = attention(b, b.pool, b.q, dev="cuda")
        close((batch.prompt_attention if form == "prompt" else batch.prefix_attention)(0, one.cuda().expand(43, 8, 128)), want, tol)


# ----------------------------------------------------------------------------------------------- as a program uses them
def step_reference(pool, rows, spans, table, prefix_pages, prefix_len, freq, gains, D, H, Hk, page, dtype):
    """One layer's append + attention in 64 bits on a host pool; q, K and V rounded to the cache's type as the cache holds them."""
    q, k, v = rows
    out = torch.zeros(q.shape[0], H, D, dtype=F64)
    at = 0
    for i, (n, l) in enumerate(spans):
        own = torch.arange(l - n, l)
        sl = slice(at, at + n)
        yq, _ = finish_heads(q[sl], own + prefix_len, freq, False, gains[0], 1e-5)
        yk, _ = finish_heads(k[sl], own + prefix_len, freq, False, gains[1], 1e-5)
        yq = yq.to(dtype).to(F64)
        for j in range(n):
            pool[table[i, own[j] // page], 0, 0, :, own[j] % page] = yk[j].to(dtype).to(F64)
            pool[table[i, own[j] // page], 0, 1, :, own[j] % page] = v[at + j].to(F64)
        t, p = torch.arange(prefix_len), torch.arange(l)
        pg, slot = torch.cat([prefix_pages[t // page], table[i, p // page]]).long(), torch.cat([t % page, p % page])
        K, V = (pool[pg, 0, j, :, slot].repeat_interleave(H // Hk, dim=1) for j in range(2))
        s = torch.einsum("rhd,nhd->hrn", yq, K) * D ** -0.5
        s = s.masked_fill(torch.arange(prefix_len + l)[None, None] > (own + prefix_len)[None, :, None], -float("inf"))
        out[sl] = torch.einsum("hrn,nhd->rhd", torch.softmax(s, -1), V)
        at += n
    return out


@pytest.mark.parametrize("dt,D", [(BF16, 128), (F16, 64), (F32, 64)])
def test_prompts_then_decoding_steps_behind_a_shared_prefix(dt, D):
    """A shared prompt is appended as one sequence, becomes the prefix of three continuations whose own prompts follow, and
    two decoding steps run: append and attention of one layer, against 64 bits all the way."""
    from paper_2410_06916_b200 import PagedKV, RowBatch, rope_table
    H, Hk, page, P0 = 8, 2, 16, 75
    own_prompt, B = [5, 33, 1], 3
    g = torch.Generator().manual_seed(9)
    n_pages = 40
    pool = torch.full((n_pages, 1, 2, Hk, page, D), float("nan")).to(dt).cuda()
    ref_pool = torch.zeros(pool.shape, dtype=F64)
    perm = torch.randperm(n_pages, generator=g).to(torch.int32)
    prefix_pages, table = perm[:5].clone(), perm[5:5 + 3 * 4].view(3, 4).clone()
    kvc, rope, freq = PagedKV(pool), rope_table(512, D), frequencies(D)
    gains = 1 + 0.1 * torch.randn(2, D, generator=g)
    gd = gains.cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")

    def layer(batch, T, form):
        x = [torch.randn(T, h, D, generator=g).to(dt) for h in (H, Hk, Hk)]
        q = batch.append(0, *(t.cuda() for t in x), rope=rope, q_gain=gd[0], k_gain=gd[1])
        return x, (batch.prompt_attention(0, q) if form == "prompt" else batch.prefix_attention(0, q))

    def check(x, got, spans, tbl, plen):
        want = step_reference(ref_pool, x, spans, tbl, prefix_pages, plen, freq, gains, D, H, Hk, page, dt)
        # q and K may round to a neighbour of the reference's rounding: a whole step each (2 h) of the scores' terms, which
        # for normed q and K are at most sqrt(D) * max |gain|^2 in all; plus the attention's own bound with |v| <= 6
        h = half_step(dt)
        s_off = 4 * h * D ** 0.5 * float(gains.abs().max()) ** 2
        close(got, want, torch.full_like(want, (2 * s_off + 4 * h) * 6.0))

    first = RowBatch(kvc, i32([0, P0]), i32([P0]), prefix_pages[None].cuda(), n_rows=P0)
    x, got = layer(first, P0, "prompt")
    check(x, got, [(P0, P0)], prefix_pages[None], 0)
    T = sum(own_prompt)
    start = [0, 5, 38, 39]
    cont = RowBatch(kvc, i32(start), i32(own_prompt), table.cuda(), n_rows=T, prefix_pages=prefix_pages.cuda(), prefix_len=P0)
    x, got = layer(cont, T, "prompt")
    check(x, got, [(n, n) for n in own_prompt], table, P0)
    lens = own_prompt
    for _ in range(2):
        lens = [l + 1 for l in lens]
        step = RowBatch(kvc, i32([0, 1, 2, 3]), i32(lens), table.cuda(), n_rows=3, max_rows=1, prefix_pages=prefix_pages.cuda(), prefix_len=P0)
        x, got = layer(step, 3, "prefix")
        check(x, got, [(1, l) for l in lens], table, P0)


@pytest.mark.parametrize("rows,dt", [(1, BF16), (40, F16)])
def test_captured_steps_follow_their_tensors(rows, dt):
    """append, prompt and prefix attention in one graph, replayed with other lengths, pages and row starts; two such graphs
    replayed side by side on two streams."""
    from paper_2410_06916_b200 import PagedKV, RowBatch, rope_table
    B, H, Hk, D, page = 3, 8, 2, 128, 16
    torch.manual_seed(3)
    rope = rope_table(600, D)
    made = []
    for j in range(2):
        b = Batch([rows] * B, [200, 90, 150], H, Hk, D, page, dt, prefix_len=100, seed=j)
        pool, batch = setup(b, max_rows=rows + 1)                    # some turns give a sequence one row more
        x = [torch.randn(b.n_rows, h, D, device="cuda").to(dt) for h in (H, Hk, Hk)]
        made.append([b, pool, batch, x])
    graphs = []
    for b, pool, batch, x in made:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            q = batch.append(0, *x, rope=rope)
            batch.prompt_attention(0, q), batch.prefix_attention(0, q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q = batch.append(0, *x, rope=rope)
            outs = [q, batch.prompt_attention(0, q), batch.prefix_attention(0, q)]
        graphs.append((g, outs))
    streams = [torch.cuda.Stream() for _ in made]
    for turn in range(3):
        for j, (b, pool, batch, x) in enumerate(made):
            row_start, kv_len, table, _ = batch._keep
            kv_len.copy_(torch.tensor([200 - 30 * turn, 90 + turn, rows + turn], dtype=torch.int32))
            row_start.copy_(torch.tensor([0, rows - (turn > 0 and rows > 1), 2 * rows - turn % 2, 3 * rows - turn % 2], dtype=torch.int32))
            if turn == 2:
                table.copy_(table.flip(0))
                kv_len.copy_(torch.tensor([rows, 90, 150], dtype=torch.int32))
            for t in x:
                t.normal_()
        torch.cuda.synchronize()
        start = made[0][2]._keep[0].tolist()
        eager = []
        for b, pool, batch, x in made:
            keep = pool.clone()
            q = batch.append(0, *x, rope=rope)
            eager.append([q, batch.prompt_attention(0, q), batch.prefix_attention(0, q), pool.clone()])
            pool.copy_(keep)
        torch.cuda.synchronize()
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                for _ in range(4):
                    g.replay()
        torch.cuda.synchronize()
        for (g, outs), want, (b, pool, _, _) in zip(graphs, eager, made):
            for name, o, w in zip(("append", "prompt", "prefix"), outs, want):
                o, w = o[:start[-1]], w[:start[-1]]
                assert torch.isfinite(w).all(), (turn, name, (~torch.isfinite(w)).nonzero()[:5].tolist())
                assert torch.equal(o, w), (turn, name, (o != w).nonzero()[:5].tolist(), float((o - w).abs().max()))
            assert torch.equal(torch.nan_to_num(pool, nan=-1.0), torch.nan_to_num(want[3], nan=-1.0))


def test_a_process_may_capture_its_first_calls():
    """No warm-up: kernels, attributes and tensor maps are set up inside the capture."""
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    code = """
import sys
sys.path[:0] = [%r, %r]
import torch
from paged_reference import Batch, attention
from test_paged_gpu import close, setup
from paper_2410_06916_b200 import rope_table
b = Batch([40, 3], [50, 60], 8, 2, 128, 16, torch.bfloat16, prefix_len=300)
pool, batch = setup(b)
want, tol = attention(b, b.pool, b.q, dev="cuda")
q = b.q.cuda()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    t, x, y = rope_table(400, 128), batch.prompt_attention(0, q), batch.prefix_attention(0, q)
g.replay()
torch.cuda.synchronize()
close(x, want, tol)
close(y, want, tol)
print("fine")
""" % (here, os.path.dirname(here))
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "fine" in done.stdout, done.stderr[-2000:]


def test_calls_side_by_side_on_two_streams():
    """Eager calls of two batches on two streams at once: nothing is shared but the code."""
    made = []
    for seed in range(2):
        b = Batch([600, 33, 1], [700, 500, 900], 16, 4, 128, 16, BF16, prefix_len=200, seed=seed)
        pool, batch = setup(b)
        q = b.q.cuda()
        made.append((pool, batch, q, batch.prompt_attention(0, q), batch.prefix_attention(0, q), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for j, (_, batch, q, _, _, s) in enumerate(made):
            got[j] += [(batch.prompt_attention(0, q, stream=s), batch.prefix_attention(0, q, stream=s))]
    torch.cuda.synchronize()
    for j, (_, _, _, p, x, _) in enumerate(made):
        for a, c in got[j]:
            assert torch.equal(a, p) and torch.equal(c, x)


def test_calls_on_a_given_stream_and_sync():
    from paper_2410_06916_b200 import batch_sync, rope_table
    b = Batch([30, 1], [30, 100], 8, 2, 128, 16, BF16, prefix_len=64)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    q = b.q.cuda()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    a, c = batch.prompt_attention(0, q, stream=s), batch.prefix_attention(0, q, stream=s)
    t = rope_table(40, 64, stream=s)
    batch_sync(stream=s)
    close(a, want, tol)
    close(c, want, tol)
    assert torch.equal(t, rope_table(40, 64))
    batch_sync()


def test_python_refusals():
    from paper_2410_06916_b200 import PagedKV, RowBatch, SwiftError, rope_table
    b = Batch([3, 2], [3, 9], 4, 2, 64, 16, BF16)
    (start, kv, table), kw = b.device_args()
    cache = PagedKV(b.pool.cuda())
    batch = RowBatch(cache, start, kv, table, **kw)
    q = b.q.cuda()
    k = q[:, :2].contiguous()
    with pytest.raises(ValueError):
        PagedKV(b.pool.cuda()[:, 0])
    with pytest.raises(ValueError):
        PagedKV(b.pool.cuda().transpose(3, 4))
    with pytest.raises(TypeError):
        RowBatch(cache, start.long(), kv, table, **kw)
    with pytest.raises(ValueError):
        RowBatch(cache, start[:-1], kv, table, **kw)
    with pytest.raises(ValueError):
        RowBatch(cache, start, kv, table, n_rows=5, prefix_pages=table[0].contiguous(), prefix_len=1000)
    with pytest.raises(ValueError):
        RowBatch(cache, start.cpu(), kv, table, **kw)
    for call in (batch.prompt_attention, batch.prefix_attention):
        with pytest.raises(ValueError):
            call(0, q[:-1])
        with pytest.raises(TypeError):
            call(0, q.half())
        with pytest.raises(ValueError):
            call(0, q.cpu())
        with pytest.raises(SwiftError, match="EINVAL"):
            call(1, q)
        with pytest.raises(SwiftError, match="EINVAL"):
            call(0, q[:, :3])
        with pytest.raises(SwiftError, match="EINVAL"):
            call(0, q, scale=-1.0)
        with pytest.raises(ValueError):
            call(0, q, out=q.float())
    with pytest.raises(TypeError):
        batch.append(0, q, k.float(), k)
    with pytest.raises(ValueError):
        batch.append(0, q, k[:, :1], k)
    with pytest.raises(ValueError):
        batch.append(0, q, k, k, rope=rope_table(8, 128))
    with pytest.raises(ValueError):
        batch.append(0, q, k, k, q_gain=torch.ones(32, device="cuda"))
    with pytest.raises(SwiftError, match="EINVAL"):
        batch.append(7, q, k, k)
