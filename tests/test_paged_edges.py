"""The paged-batch operators at the edges of what their interface allows: plans that reach further than their tables, scores
that are not finite or far from zero, waits that run out, tensors of other streams (bounds as in paged_reference.py)."""
import pytest
import torch

from paged_reference import F64, Batch, append_tolerance, attention, finish_heads, frequencies, half_step
from test_paged_gpu import close, setup

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def call(batch, form):
    return batch.prompt_attention if form == "prompt" else batch.prefix_attention


# ----------------------------------------------------------------------------------------------- plans that reach too far
class Long(Batch):
    """A batch whose kv_len reach beyond the page table: the positions behind it hold nothing."""
    def longer(self, kv):
        self.capacity = self.page_table.shape[1] * self.page
        self.kv = kv
        return self

    def visible(self, i):
        kv, self.kv = self.kv, [min(max(l, 0), self.capacity) for l in self.kv]
        try:
            return super().visible(i)
        finally:
            self.kv = kv


@pytest.mark.gpu
@pytest.mark.parametrize("dt,x_dtype,dim,heads", [(BF16, BF16, 128, 8), (F16, F32, 64, 4), (F32, F32, 34, 2)])
def test_append_leaves_out_rows_behind_the_page_table(dt, x_dtype, dim, heads):
    """kv_len one, three and 2^31 - 1 beyond a full table, just full, below zero: rows keep their positions, and of those behind
    the table nothing is written."""
    from paper_2410_06916_b200 import PagedKV, RowBatch, rope_table
    page, width, B = 16, 4, 7
    cap = page * width
    n = [1, 3, 5, 2, 4, 2, 1]
    kv = [cap + 1, cap + 3, cap + 3, cap, (1 << 31) - 1, -3, 40]
    T, kv_heads = sum(n), 2
    g = torch.Generator().manual_seed(2)
    x = [torch.randn(T, h, dim, generator=g).to(x_dtype) for h in (heads, kv_heads, kv_heads)]
    start = [0]
    for a in n:
        start.append(start[-1] + a)
    table = torch.randperm(B * width, generator=g).to(torch.int32).view(B, width)
    before = torch.randn(B * width, 1, 2, kv_heads, page, dim, generator=g).to(dt)
    pool = before.cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    batch = RowBatch(PagedKV(pool), i32(start), i32(kv), table.cuda(), n_rows=T)
    out = torch.full((T, heads, dim), 3.0, device="cuda", dtype=dt)
    xd = [t.cuda() for t in x]
    batch.append(0, *xd, rope=rope_table(2 * cap, dim), out=out)
    want_pool, tol_pool = before.to(F64), torch.zeros(before.shape, dtype=F64)
    want_q, tol_q = torch.full((T, heads, dim), 3.0, dtype=F64), torch.zeros(T, heads, dim, dtype=F64)
    written = 0
    for i in range(B):
        for j in range(n[i]):
            own, row = kv[i] - n[i] + j, start[i] + j
            if not 0 <= own < cap:
                continue
            written += 1
            pos = torch.tensor([own])
            (yq, mq), (yk, mk) = (finish_heads(t[row:row + 1], pos, frequencies(dim), False, None, 1e-5) for t in x[:2])
            want_q[row], tol_q[row] = yq[0], append_tolerance(yq, mq, dim, dt)[0]
            at = int(table[i, own // page])
            want_pool[at, 0, 0, :, own % page], tol_pool[at, 0, 0, :, own % page] = yk[0], append_tolerance(yk, mk, dim, dt)[0]
            v = x[2][row].to(F64)
            want_pool[at, 0, 1, :, own % page], tol_pool[at, 0, 1, :, own % page] = v, half_step(dt) * v.abs() + (2.0 ** -25 if dt == F16 else 0.0)
    assert written == 2 + 2 + 1
    close(out, want_q, tol_q)
    close(pool, want_pool, tol_pool)


LONG = [
    # rows, cached (the first fills the table), beyond, heads, kv heads, dim, type, prefix
    ([1, 1, 1], [64, 20, 64], [65, 20, 70], 8, 2, 128, BF16, 0),
    ([5, 9, 3], [64, 64, 30], [66, 67, 30], 8, 2, 128, F16, 100),
    ([9, 9, 9], [640, 640, 30], [641, 700, 30], 14, 2, 64, BF16, 700),
    ([40, 130, 50], [512, 512, 300], [530, 513, 300], 8, 2, 128, BF16, 0),
    ([40, 130, 50], [512, 512, 300], [530, 800, 300], 4, 4, 96, F16, 90),
    ([40, 5, 50], [512, 512, 300], [530, 514, -7], 4, 2, 36, F32, 90),
    ([700, 650], [704, 704], [720, 710], 8, 8, 64, F32, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", LONG, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c[3:]))
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_attention_keeps_the_positions_of_sequences_beyond_their_table(case, form):
    n, kv, longer, H, Hk, dim, dt, prefix = case
    b = Long(n, kv, H, Hk, dim, 16, dt, prefix_len=prefix).longer(longer)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    close(call(batch, form)(0, b.q.cuda()), want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("each,dt", [(4, BF16), (60, BF16), (4, F32)])
def test_row_starts_behind_the_packed_rows_move_no_row(form, each, dt):
    """The last sequence claims two rows more than the tensors have: its first rows stay at their positions."""
    from paper_2410_06916_b200 import PagedKV, RowBatch
    b = Batch([each, each], [200, 170], 8, 2, 64, 16, dt)
    (start, kv, table), kw = b.device_args()
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    pool = b.pool.cuda()
    kw["n_rows"] -= 2
    batch = RowBatch(PagedKV(pool), start, kv, table, **kw)
    q = b.q[:-2].cuda()
    close(call(batch, form)(0, q), want[:-2], tol[:-2])
    k = torch.randn(2 * each - 2, 2, 64, device="cuda").to(dt)
    before = pool.clone()
    batch.append(0, q, k, k)
    for i in range(2):
        for j in range(each):
            own, row = b.kv[i] - each + j, i * each + j
            at = (int(b.page_table[i, own // 16]), 0, slice(None), slice(None), own % 16)
            before[at] = k[row] if row < len(k) else before[at]
    assert torch.equal(torch.nan_to_num(pool, nan=-1.0), torch.nan_to_num(before, nan=-1.0))


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("each,dt,prefix", [(1, BF16, 0), (4, F16, 0), (4, BF16, 50), (60, BF16, 0), (3, F32, 0)])
def test_a_sequence_that_claims_every_row_there_can_be(form, each, dt, prefix):
    """row_start ends at 2^31 - 1: the rows that exist lie far before the sequence's first position and see the prefix alone."""
    from paper_2410_06916_b200 import PagedKV, RowBatch
    b = Batch([each, each], [200, 700], 8, 2, 64, 16, dt, prefix_len=prefix)
    (start, kv, table), kw = b.device_args()
    start[2] = (1 << 31) - 1
    got = call(RowBatch(PagedKV(b.pool.cuda()), start, kv, table, **kw), form)(0, b.q.cuda())
    b.kv[1] = 0
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    assert prefix or not want[each:].any()
    close(got, want, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["prompt", "prefix"])
@pytest.mark.parametrize("each,dt", [(4, BF16), (60, F16), (3, F32)])
def test_lengths_below_zero_and_row_starts_that_descend(form, each, dt):
    """A length below zero is an empty cache: such rows see nothing and append nothing.  Row starts that descend hold no rows."""
    from paper_2410_06916_b200 import PagedKV, RowBatch
    b = Batch([each, each], [200, 170], 8, 2, 64, 16, dt)
    (start, kv, table), kw = b.device_args()
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    pool, q = b.pool.cuda(), b.q.cuda()
    before = pool.clone()
    batch = RowBatch(PagedKV(pool), start, torch.tensor([200, -3], dtype=torch.int32, device="cuda"), table, **kw)
    got = call(batch, form)(0, q)
    close(got[:each], want[:each], tol[:each])
    assert (got[each:] == 0).all()
    rows = torch.full_like(q, 2.0)
    k = torch.ones(2 * each, 2, 64, device="cuda", dtype=dt)
    assert (batch.append(0, q, k, k, out=rows)[each:] == 2).all()
    own = set(range(200 - each, 200))
    for p in range(200):
        at = (int(b.page_table[0, p // 16]), 0, slice(None), slice(None), p % 16)
        before[at] = 1.0 if p in own else before[at]
    assert torch.equal(torch.nan_to_num(pool, nan=-1.0), torch.nan_to_num(before, nan=-1.0))
    backwards = torch.tensor([2 * each, each, -2], dtype=torch.int32, device="cuda")
    batch = RowBatch(PagedKV(pool), backwards, kv, table, **kw)
    out = torch.full_like(q, 9.0)
    call(batch, form)(0, q, out=out)
    batch.append(0, q, k + 1, k + 1, out=rows.fill_(9.0))
    assert (out == 9).all() and (rows == 9).all()
    assert torch.equal(torch.nan_to_num(pool, nan=-1.0), torch.nan_to_num(before, nan=-1.0))


# ----------------------------------------------------------------------------------------------- waits that run out
WAITS = [
    # rows of each of four sequences, cached, heads, kv heads, dim, type, prefix, form
    (130, 500, 8, 2, 128, BF16, 0, "prompt"), (3, 300, 4, 4, 64, F16, 40, "prompt"),
    (1, 3000, 8, 2, 128, BF16, 0, "prefix"), (2, 700, 8, 2, 64, F16, 500, "prefix"),            # the few-row kernel, its prefix too
    (9, 900, 14, 2, 128, F16, 2000, "prefix"),                                                 # ... beside the many-row kernel
    (40, 100, 8, 1, 128, BF16, 20000, "prefix"),                                                # the many-row kernel alone
]


def waits_run_out(case):
    """In a process of its own: the probe gives up, the report comes once, the next call on the same workspace is right."""
    import ctypes as C
    import time
    from paper_2410_06916_b200 import SwiftError, batch_sync, lib
    from paper_2410_06916_b200.binding import _DevBuf
    each, kv, H, Hk, dim, dt, prefix, form = case
    b = Batch([each] * 4, [kv, kv - 9, kv // 2, kv], H, Hk, dim, 16, dt, prefix_len=prefix)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    q = b.q.cuda()
    rows = 0 if form == "prompt" else batch.max_rows
    need = lib().swift_prefix_workspace_bytes(C.byref(batch.kv._c), C.byref(batch._c), H, max(rows, 1))
    out = torch.empty_like(q)
    a = batch._attention(0, q, None)
    a.out = out.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    for fill in (0, 0x7F, 0xFF, 0x01):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")       # what an entry no one wrote may hold
        where = _DevBuf(ws.data_ptr(), need)
        torch.cuda.synchronize()
        t0 = time.monotonic()
        assert lib().swift_probe_batch_wait_limit(C.byref(batch.kv._c), C.byref(batch._c), C.byref(a), rows, where, 1000, stream) == 0
        try:
            batch_sync()
            raise AssertionError("no report")
        except SwiftError as e:
            assert "ETIMEOUT" in str(e), e
        assert time.monotonic() - t0 < 5.0
        batch_sync()
        if form == "prefix":
            assert lib().swift_prefix_attention(C.byref(batch.kv._c), C.byref(batch._c), C.byref(a), rows, where, stream) == 0
        else:
            assert lib().swift_prompt_attention(C.byref(batch.kv._c), C.byref(batch._c), C.byref(a), stream) == 0
        batch_sync()
        close(out, want, tol)


def in_its_own_process(function, *args):
    """Runs a function of this file in a fresh process: what it leaves behind on the device is no other test's."""
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    code = (f"import sys; sys.path[:0] = [{here!r}, {os.path.dirname(here)!r}]\nimport torch\nimport test_paged_edges as t\n"
            f"t.{function}(*{args!r})\ntorch.cuda.synchronize()\nprint('fine')\n")
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "fine" in done.stdout, done.stderr[-2000:]


def every_stream_is_told():
    """A wait that runs out is reported once to every stream that asks, whoever asks first, and to threads side by side."""
    import ctypes as C
    import threading
    from paper_2410_06916_b200 import SwiftError, batch_sync, lib
    from paper_2410_06916_b200.binding import _DevBuf
    b = Batch([40], [300], 8, 2, 128, 16, BF16)
    pool, batch = setup(b)
    q = b.q.cuda()
    out = torch.empty_like(q)
    a = batch._attention(0, q, None)
    a.out = out.data_ptr()
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()

    def told(s):
        try:
            batch_sync(stream=s)
            return False
        except SwiftError as e:
            assert "ETIMEOUT" in str(e), e
            return True
    assert not any(told(s) for s in streams)
    for _ in range(3):
        assert lib().swift_probe_batch_wait_limit(C.byref(batch.kv._c), C.byref(batch._c), C.byref(a), 0, _DevBuf(None, 0), 500,
                                                  streams[1].cuda_stream) == 0
        streams[1].synchronize()
        got = [None] * 4
        threads = [threading.Thread(target=lambda i=i: got.__setitem__(i, told(streams[i]))) for i in range(4)]
        [t.start() for t in threads], [t.join() for t in threads]
        assert got == [True] * 4, got
        assert not any(told(s) for s in streams)
    assert told(torch.cuda.current_stream())                             # its first report
    assert not told(torch.cuda.current_stream())


@pytest.mark.gpu
def test_a_report_takes_nothing_from_other_streams():
    in_its_own_process("every_stream_is_told")


@pytest.mark.gpu
@pytest.mark.parametrize("case", WAITS, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_a_wait_that_runs_out_is_a_status(case):
    """Copies that are never asked for: every block gives up within its limit, swift_batch_sync reports it once, and entries
    of the workspace that were never written lead nowhere."""
    in_its_own_process("waits_run_out", case)


def test_the_wait_probe_refuses_what_has_no_waits():
    import ctypes as C
    from paper_2410_06916_b200 import lib, paged
    from paper_2410_06916_b200.binding import _DevBuf
    at = 1 << 20
    batch = paged._Batch(2, 4, at, at, at, 4, None, 0)
    args = paged._Attention(0, 4, paged._Rows(at, 256, 64), 0.125, at)
    probe = lambda dtype, rows, ws, us: lib().swift_probe_batch_wait_limit(
        C.byref(paged._Kv(at, dtype, 8, 1, 2, 16, 64)), C.byref(batch), C.byref(args), rows, ws, us, None)
    ws = _DevBuf(at, 1 << 40)
    assert probe(0, 4, ws, 100) == 6 and probe(0, 0, ws, 100) == 6
    assert probe(1, 4, ws, 0) == 1 and probe(1, 4, ws, 100001) == 1 and probe(1, -1, ws, 100) == 1
    assert probe(1, 4, _DevBuf(at, 16), 100) == 3 and probe(1, 4, _DevBuf(None, 0), 100) == 1


# ----------------------------------------------------------------------------------------------- scores that are not finite
SHAPES = [
    # rows of each of two sequences, cached, heads, kv heads, dim, type, prefix: every kernel and form
    (130, 400, 8, 2, 128, BF16, 0), (130, 400, 8, 2, 64, F16, 0),               # many rows
    (40, 300, 8, 2, 128, F16, 300), (24, 300, 8, 1, 128, BF16, 2000),           # ... and a shared prefix
    (3, 300, 8, 2, 128, BF16, 0), (9, 300, 8, 2, 64, F16, 0),                   # few rows
    (200, 400, 8, 8, 36, F16, 0), (3, 200, 8, 2, 64, F32, 0),                   # fp32 arithmetic
]
SHAPE_IDS = lambda s: "-".join(str(x).replace("torch.", "") for x in s) if isinstance(s, tuple) else str(s)


def edge_batch(shape):
    each, kv, H, Hk, dim, dt, prefix = shape
    b = Batch([each, each], [kv, kv - 7], H, Hk, dim, 32, dt, prefix_len=prefix)
    b.q[:, :, 0] = b.q[:, :, 0].abs() + 0.25
    return b


def key_slot(b, i, p, head):
    """Index of own position p of sequence i in K of a kv head, all dims."""
    return int(b.page_table[i, p // b.page]), b.block, 0, head, p % b.page


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_a_visible_key_without_a_finite_score_shows_wherever_it_lies(form, shape, value):
    """One dim of one cached key of sequence 0 is NaN or infinite, at 32 positions in turn that every row sees: the rows of its
    group are NaN in every dim, those of the other sequence and the other kv head stay what they were."""
    b = edge_batch(shape)
    pool, batch = setup(b)
    q, each, G = b.q.cuda(), b.n[0], b.heads // b.kv_heads
    clean = call(batch, form)(0, q)
    assert torch.isfinite(clean).all()
    for p in range(64, 96):
        at = key_slot(b, 0, p, 0)
        was = pool[at].clone()
        pool[at][0] = value
        got = call(batch, form)(0, q)
        pool[at] = was
        assert torch.isnan(got[:each, :G]).all(), p
        assert torch.equal(got[each:], clean[each:]) and torch.equal(got[:each, G:], clean[:each, G:]), p


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_scores_of_minus_infinity_weigh_nothing(form, shape):
    """Keys whose score is -infinity (a whole page of them, its first and last keys next to finite ones) count as hidden; rows that
    see no other key give 0, as rows that see nothing."""
    b = edge_batch(shape)
    pool, batch = setup(b)
    q = b.q.cuda()
    hidden = edge_batch(shape)
    hidden.page_table[0, 2] = hidden.n_pages
    want, tol = attention(hidden, b.pool, b.q, dev="cuda")
    low = -float("inf")
    for p in range(64, 96):
        for h in range(b.kv_heads):
            pool[key_slot(b, 0, p, h)][0] = low
    close(call(batch, form)(0, q), want, tol)
    if b.prefix_len == 0:
        for p in range(b.kv[0]):
            pool[key_slot(b, 0, p, 0)][0] = low
        got, G = call(batch, form)(0, q), b.heads // b.kv_heads
        assert (got[:b.n[0], :G] == 0).all()
        close(got[b.n[0]:], want[b.n[0]:], tol[b.n[0]:])
        close(got[:b.n[0], G:], want[:b.n[0], G:], tol[:b.n[0], G:])


# ----------------------------------------------------------------------------------------------- scores far from zero
@pytest.mark.gpu
@pytest.mark.parametrize("scale", [None, 0.0371, 0.31, 0.77])
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("form", ["prompt", "prefix"])
def test_scores_far_from_zero(form, shape, scale):
    """q and K hold +-2^14 (fp32, bf16: +-2^17), so that every product and every partial sum of a score is at most 128 times 2^28
    (2^34): exact in fp32 in any order.  Two scores are equal or at least 2^29 (2^35) times the scale apart, so the exact
    weights are equal for the keys with a row's highest score and below 2^-1000 for all others: the result is the mean of those
    keys' V.  Errors: the weights' common factor cancels but for their rounding (2 h) and that of sums of N terms (2 N u), and
    the result is rounded once (h)."""
    b = edge_batch(shape)
    g = torch.Generator().manual_seed(11)
    big = 2.0 ** (14 if b.dtype == F16 else 17)
    signs = lambda t: torch.where(torch.rand(t.shape, generator=g) < 0.5, -big, big).to(t.dtype)
    b.q[:] = signs(b.q)
    b.pool[:, :, 0] = torch.where(torch.isnan(b.pool[:, :, 0]), b.pool[:, :, 0], signs(b.pool[:, :, 0]))
    pool, batch = setup(b)
    got = call(batch, form)(0, b.q.cuda(), scale=scale).to(F64).cpu()
    G, h, u = b.heads // b.kv_heads, half_step(b.dtype), 2.0 ** -24
    assert torch.isfinite(got).all()
    for i, n in enumerate(b.n):
        page, slot, own = (torch.tensor([x[j] for x in b.visible(i)]) for j in range(3))
        kv = b.pool[page, b.block, :, :, slot].to(F64)
        k, v = (kv[:, j].repeat_interleave(G, dim=1) for j in range(2))
        s = torch.einsum("rhd,nhd->hrn", b.q[b.start[i]:b.start[i] + n].to(F64), k)
        last = torch.arange(n) + (b.kv[i] - n)
        s = s.masked_fill(((own[None] >= 0) & (own[None] > last[:, None]))[None], -float("inf"))
        best = (s == s.amax(-1, keepdim=True)).to(F64)
        want, size = (torch.einsum("hrn,nhd->rhd", best, x) / best.sum(-1).T[..., None] for x in (v, v.abs()))
        close(got[b.start[i]:b.start[i] + n], want, h * want.abs() + (2 * h + 2 * len(page) * u) * size)


# ----------------------------------------------------------------------------------------------- tensors of other streams
@pytest.mark.gpu
def test_tensors_freed_behind_a_call_on_another_stream_stay_until_it_is_done():
    """Everything a call takes is dropped right behind it and its sizes are asked for again on the tensors' own stream, while the
    given stream still waits in front of the call: the call reads and writes what it was given."""
    from paper_2410_06916_b200 import PagedKV, RowBatch, rope_table
    b = Batch([70, 5], [200, 150], 8, 2, 128, 16, BF16, prefix_len=40)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    g = torch.Generator().manual_seed(3)
    host = [b.q] + [torch.randn(75, 2, 128, generator=g).to(BF16) for _ in range(2)]
    gain = 1 + 0.1 * torch.randn(128, generator=g)
    rope = rope_table(300, 128)
    s = torch.cuda.Stream()

    def fresh():
        (start, kv, table), kw = b.device_args()
        pool = b.pool.cuda()
        return pool, RowBatch(PagedKV(pool), start, kv, table, **kw)

    def overwrite(sizes):
        return [torch.full((n,), 0x7B, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]

    def nbytes(*tensors):
        return [t.numel() * t.element_size() for t in tensors]
    pool, batch = fresh()
    plain = batch.append(0, *(t.cuda() for t in host), rope=rope, q_gain=gain.cuda(), k_gain=gain.cuda()), pool.clone()
    for form in ("prompt", "prefix", "append"):
        pool, batch = fresh()
        x, gains = [t.cuda() for t in host], gain.cuda()
        sizes = nbytes(*x, gains, *batch._keep)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(40_000_000)                                # about 20 ms
        if form == "append":
            table = rope.clone()
            s.wait_stream(torch.cuda.current_stream())
            sizes += nbytes(table)
            got = batch.append(0, *x, rope=table, q_gain=gains, k_gain=gains, stream=s)
            del table
        else:
            got = call(batch, form)(0, x[0], stream=s)
            sizes += nbytes(pool)
        assert not s.query()
        kept = pool if form == "append" else None
        del x, gains, pool, batch
        taken = overwrite(sizes)
        torch.cuda.synchronize()
        if form == "append":
            assert torch.equal(got, plain[0]) and torch.equal(torch.nan_to_num(kept, nan=-1.0), torch.nan_to_num(plain[1], nan=-1.0))
        else:
            close(got, want, tol)
        del taken, kept, got


# ----------------------------------------------------------------------------------------------- refusals of the torch side
@pytest.mark.gpu
def test_tensors_that_require_gradients_are_refused():
    """No call has a backward pass: what autograd would follow is refused, and taken under no_grad."""
    from paper_2410_06916_b200 import rope_table
    b = Batch([3, 2], [3, 9], 4, 2, 64, 16, BF16)
    pool, batch = setup(b)
    q = b.q.cuda()
    k = q[:, :2].contiguous()
    rope, gain = rope_table(16, 64), torch.ones(64, device="cuda")
    leaf = lambda t: t.clone().requires_grad_()
    calls = [lambda: batch.append(0, leaf(q), k, k), lambda: batch.append(0, q, leaf(k), k), lambda: batch.append(0, q, k, leaf(k)),
             lambda: batch.append(0, q, k, k, q_gain=leaf(gain)), lambda: batch.append(0, q, k, k, k_gain=leaf(gain)),
             lambda: batch.append(0, q, k, k, rope=leaf(rope)), lambda: batch.append(0, q, k, k, out=leaf(q)),
             lambda: batch.append(0, leaf(q.float()) * 1.0, k.float(), k.float()),
             lambda: batch.prompt_attention(0, leaf(q)), lambda: batch.prefix_attention(0, leaf(q)),
             lambda: batch.prompt_attention(0, q, out=leaf(q)), lambda: batch.prefix_attention(0, q, out=leaf(q)),
             lambda: rope_table(16, 64, out=leaf(rope))]
    before = pool.clone()
    for f in calls:
        with pytest.raises(ValueError, match="gradient"):
            f()
    assert torch.equal(torch.nan_to_num(pool, nan=-1.0), torch.nan_to_num(before, nan=-1.0))
    with torch.no_grad():
        for f in calls:
            assert not f().requires_grad or f is calls[6] or f in calls[10:]
    with torch.inference_mode():
        assert torch.equal(batch.prompt_attention(0, q), batch.prompt_attention(0, leaf(q)))


@pytest.mark.parametrize("kw", [dict(n_positions=(1 << 32) + 8), dict(n_positions=1 << 31), dict(rotary_dim=(1 << 32) + 64),
                                dict(original_positions=1 << 32), dict(n_positions=-(1 << 32) + 8)], ids=str)
def test_numbers_beyond_32_bits_are_refused(kw):
    """... rather than cut to their low bits: a table of 2^32 + 8 positions had 8."""
    from paper_2410_06916_b200 import rope_table
    args = dict(n_positions=8, rotary_dim=64, device="cuda:0")
    args.update(kw)
    with pytest.raises(ValueError, match="32 bits"):
        rope_table(**args)


@pytest.mark.gpu
def test_blocks_and_lengths_beyond_32_bits_are_refused():
    from paper_2410_06916_b200 import PagedKV, RowBatch
    b = Batch([3, 2], [3, 9], 4, 2, 64, 16, BF16)
    pool, batch = setup(b)
    q = b.q.cuda()
    k = q[:, :2].contiguous()
    for f in (lambda x: batch.append(x, q, k, k), lambda x: batch.prompt_attention(x, q), lambda x: batch.prefix_attention(x, q)):
        for block in (1 << 32, -(1 << 32), 1 << 31):
            with pytest.raises(ValueError, match="32 bits"):
                f(block)
    (start, kv, table), kw = b.device_args()
    for more in (dict(n_rows=(1 << 32) + 5), dict(prefix_len=1 << 32, prefix_pages=table[0].contiguous())):
        with pytest.raises(ValueError):
            RowBatch(PagedKV(pool), start, kv, table, **{**kw, **more})


@pytest.mark.gpu
def test_captured_calls_on_a_given_stream_whose_inputs_are_dropped():
    """stream= inside a capture, on the capturing stream and on one forked from it, with inputs freed during the capture; the two
    graphs share one memory pool and are replayed in turn."""
    b = Batch([40, 3], [50, 60], 8, 2, 128, 16, BF16, prefix_len=300)
    pool, batch = setup(b)
    want, tol = attention(b, b.pool, b.q, dev="cuda")
    q, main, side = b.q.cuda(), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs, share = [], None
    for forked in (False, True):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=main, pool=share):
            lent = q.clone()
            on = side if forked else main
            if forked:
                side.wait_stream(main)
            got = [call(batch, form)(0, lent, stream=on) for form in ("prompt", "prefix", "prefix")]
            if forked:
                main.wait_stream(side)
            del lent
            got = [t.clone() for t in got] + [batch.prefix_attention(0, q)]
        share = g.pool()
        graphs.append((g, got))
    for _ in range(3):
        for g, got in graphs:
            g.replay()
            torch.cuda.synchronize()
            for t in got:
                close(t, want, tol)
