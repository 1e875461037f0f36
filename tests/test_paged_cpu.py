"""Refusals of the paged-batch calls and their Python side: nothing here needs a device, every call must return before it
would enqueue anything."""
import ctypes as C

import pytest
import torch

from paper_2410_06916_b200 import paged
from paper_2410_06916_b200.binding import _DevBuf, load_library

EINVAL, ECAPACITY, EUNSUPPORTED = 1, 3, 6
FAKE = 1 << 20            # an aligned address that nothing may touch


def kv(**kw):
    v = dict(pool=FAKE, dtype=1, n_pages=8, n_blocks=2, n_kv_heads=2, page_size=16, head_dim=64)
    v.update(kw)
    return paged._Kv(*v.values())


def batch(**kw):
    v = dict(n_seqs=2, n_rows=4, row_start=FAKE, kv_len=FAKE, page_table=FAKE, table_stride=4, prefix_pages=None, prefix_len=0)
    v.update(kw)
    return paged._Batch(*v.values())


def attention(**kw):
    v = dict(block=1, n_heads=4, q=paged._Rows(FAKE, 256, 64), scale=0.125, out=FAKE)
    v.update(kw)
    return paged._Attention(*v.values())


def append(**kw):
    rows = lambda h: paged._Rows(FAKE, h * 64, 64)
    a = paged._Append()
    v = dict(block=0, n_heads=4, x_dtype=1, q=rows(4), k=rows(2), v=rows(2), eps=1e-5, rope=FAKE, rope_positions=64, rotary_dim=64, q_out=FAKE)
    v.update(kw)
    for k, x in v.items():
        setattr(a, k, x)
    return a


BAD_CACHES = [dict(pool=None), dict(pool=FAKE + 8), dict(dtype=3), dict(dtype=-1), dict(n_pages=0), dict(n_blocks=0), dict(n_kv_heads=0),
              dict(page_size=4), dict(page_size=24), dict(page_size=256), dict(head_dim=0), dict(head_dim=63), dict(head_dim=258),
              dict(n_blocks=1 << 20, n_kv_heads=1024)]
BAD_BATCHES = [dict(n_seqs=-1), dict(n_rows=-1), dict(row_start=None), dict(kv_len=None), dict(page_table=None), dict(table_stride=0),
               dict(table_stride=1 << 28), dict(prefix_len=-1), dict(prefix_len=5), dict(prefix_len=(1 << 30) + 1, prefix_pages=FAKE)]
BAD_ATTENTION = [dict(block=2), dict(block=-1), dict(n_heads=0), dict(n_heads=3), dict(n_heads=8192), dict(scale=0.0), dict(scale=-1.0),
                 dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None), dict(out=FAKE + 8), dict(q=paged._Rows(None, 256, 64)),
                 dict(q=paged._Rows(FAKE + 2, 256, 64)), dict(q=paged._Rows(FAKE, 257, 64)), dict(q=paged._Rows(FAKE, 256, 4)),
                 dict(q=paged._Rows(FAKE, -256, 64))]
BAD_APPEND = [dict(block=2), dict(n_heads=-1), dict(rotary_dim=66), dict(rotary_dim=31), dict(rotary_dim=0), dict(rope=FAKE + 4),
              dict(rope_positions=-1), dict(q=paged._Rows(None, 256, 64)), dict(k=paged._Rows(None, 128, 64)), dict(v=paged._Rows(FAKE + 1, 128, 64)),
              dict(q_out=None), dict(q_out=FAKE + 1), dict(q_gain=FAKE, eps=float("nan")), dict(k_gain=FAKE, eps=-1.0), dict(q_gain=FAKE + 2),
              dict(k=paged._Rows(FAKE, -128, 64))]


def every_call(k, b, a=None, x=None):
    lib = load_library()
    a, x = a or attention(), x or append()
    ws = _DevBuf(FAKE, 1 << 40)
    return {"append": lib.swift_kv_append(C.byref(k), C.byref(b), C.byref(x), None),
            "prompt": lib.swift_prompt_attention(C.byref(k), C.byref(b), C.byref(a), None),
            "prefix": lib.swift_prefix_attention(C.byref(k), C.byref(b), C.byref(a), 4, ws, None)}


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(bad):
    assert set(every_call(kv(**bad), batch()).values()) == {EINVAL}
    assert load_library().swift_prefix_workspace_bytes(C.byref(kv(**bad)), C.byref(batch()), 4, 4) == 0


@pytest.mark.parametrize("bad", BAD_BATCHES, ids=str)
def test_bad_batches_are_refused(bad):
    assert set(every_call(kv(), batch(**bad)).values()) == {EINVAL}
    assert load_library().swift_prefix_workspace_bytes(C.byref(kv()), C.byref(batch(**bad)), 4, 4) == 0


def test_too_many_sequences_are_refused():
    assert set(every_call(kv(), batch(n_seqs=4097)).values()) == {ECAPACITY}


@pytest.mark.parametrize("bad", BAD_ATTENTION, ids=str)
def test_bad_attention_arguments_are_refused(bad):
    got = every_call(kv(), batch(), a=attention(**bad), x=append(block=9))
    assert got == {"append": EINVAL, "prompt": EINVAL, "prefix": EINVAL}
    assert load_library().swift_batch_error()


@pytest.mark.parametrize("bad", BAD_APPEND, ids=str)
def test_bad_append_arguments_are_refused(bad):
    lib = load_library()
    assert lib.swift_kv_append(C.byref(kv()), C.byref(batch()), C.byref(append(**bad)), None) == EINVAL


def test_append_takes_fp32_or_the_caches_type():
    lib = load_library()
    assert lib.swift_kv_append(C.byref(kv(dtype=1)), C.byref(batch()), C.byref(append(x_dtype=2)), None) == EUNSUPPORTED
    assert lib.swift_kv_append(C.byref(kv(dtype=0)), C.byref(batch()), C.byref(append(x_dtype=1)), None) == EUNSUPPORTED


def test_null_structures_are_refused():
    lib = load_library()
    assert lib.swift_kv_append(None, None, None, None) == EINVAL
    assert lib.swift_kv_append(C.byref(kv()), C.byref(batch()), None, None) == EINVAL
    assert lib.swift_prompt_attention(C.byref(kv()), C.byref(batch()), None, None) == EINVAL
    assert lib.swift_prefix_attention(C.byref(kv()), None, C.byref(attention()), 4, _DevBuf(FAKE, 1 << 40), None) == EINVAL
    assert lib.swift_rope_table(None, None, None) == EINVAL


def test_workspaces_that_do_not_fit_are_refused():
    lib = load_library()
    need = lib.swift_prefix_workspace_bytes(C.byref(kv()), C.byref(batch()), 4, 4)
    assert need > 0
    call = lambda ws, rows=4: lib.swift_prefix_attention(C.byref(kv()), C.byref(batch()), C.byref(attention()), rows, ws, None)
    assert call(_DevBuf(FAKE, need - 1)) == ECAPACITY
    assert call(_DevBuf(None, need)) == EINVAL
    assert call(_DevBuf(FAKE + 16, need)) == EINVAL
    assert call(_DevBuf(FAKE, need), rows=0) == EINVAL
    assert lib.swift_prefix_workspace_bytes(C.byref(kv()), C.byref(batch()), 3, 4) == 0
    assert lib.swift_prefix_workspace_bytes(C.byref(kv()), C.byref(batch()), 4, 0) == 0


def test_workspace_grows_with_what_it_holds():
    lib = load_library()
    size = lambda heads, rows, **b: lib.swift_prefix_workspace_bytes(C.byref(kv(head_dim=128)), C.byref(batch(**b)), heads, rows)
    base = size(4, 1, n_rows=64, n_seqs=64)
    assert size(32, 1, n_rows=64, n_seqs=64) >= base and size(4, 1, n_rows=4096, n_seqs=4096) >= base
    assert size(4, 1, n_rows=64, n_seqs=64, prefix_pages=FAKE, prefix_len=100000) >= base


def test_empty_batches_do_nothing():
    assert set(every_call(kv(), batch(n_seqs=0, row_start=None, kv_len=None, page_table=None)).values()) == {0}
    assert set(every_call(kv(), batch(n_rows=0)).values()) == {0}


@pytest.mark.parametrize("bad", [dict(n_positions=-1), dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=258), dict(theta=0.0),
                                 dict(theta=float("inf")), dict(factor=0.0), dict(factor=float("nan")), dict(magnitude=float("nan")),
                                 dict(original_positions=-1), dict(original_positions=10, low_turns=4.0, high_turns=4.0),
                                 dict(original_positions=10, low_turns=float("nan"))], ids=str)
def test_bad_rope_descriptions_are_refused(bad):
    v = dict(n_positions=8, rotary_dim=64, theta=1e4, factor=1.0, original_positions=0, low_turns=1.0, high_turns=4.0, magnitude=1.0)
    v.update(bad)
    assert load_library().swift_rope_table(C.byref(paged._RopeDesc(*v.values())), FAKE, None) == EINVAL
    assert load_library().swift_rope_table(C.byref(paged._RopeDesc(8, 64, 1e4, 1.0, 0, 1.0, 4.0, 1.0)), FAKE + 4, None) == EINVAL


def test_an_empty_table_is_no_work():
    assert load_library().swift_rope_table(C.byref(paged._RopeDesc(0, 64, 1e4, 1.0, 0, 1.0, 4.0, 1.0)), FAKE, None) == 0


def test_host_tensors_are_refused():
    with pytest.raises(ValueError, match="CUDA"):
        paged.PagedKV(torch.zeros(2, 1, 2, 1, 8, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="CUDA"):
        paged.rope_table(8, 64, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        paged.rope_table(8, 64, out=torch.zeros(8, 32, 2))
    with pytest.raises(ValueError, match="CUDA"):
        paged.batch_sync("cpu")
