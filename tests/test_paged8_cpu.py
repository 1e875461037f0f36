"""Refusals of the 8-bit cache's calls and of sample_rows: nothing here needs a device, every call must return before it would enqueue
anything."""
import ctypes as C

import pytest
import torch

import test_paged_cpu as wide
from paper_2410_06916_b200 import paged, sampling
from paper_2410_06916_b200.binding import _DevBuf, load_library

EINVAL, ECAPACITY, EUNSUPPORTED = 1, 3, 6
FAKE = wide.FAKE


def kv8(scales=FAKE, **kw):
    return paged._Kv8(wide.kv(**{"dtype": 3, **kw}), scales)


def append(**kw):
    return wide.append(**kw)


def every_call(k, b, a=None, x=None, x_dtype=1):
    lib = load_library()
    a, x = a or wide.attention(), x or append()
    ws = _DevBuf(FAKE, 1 << 40)
    return {"append": lib.swift_coded_append(C.byref(k), C.byref(b), C.byref(x), None),
            "prompt": lib.swift_coded_prompt_attention(C.byref(k), C.byref(b), C.byref(a), x_dtype, None),
            "prefix": lib.swift_coded_prefix_attention(C.byref(k), C.byref(b), C.byref(a), x_dtype, 4, ws, None)}


@pytest.mark.parametrize("bad", [x for x in wide.BAD_CACHES if "dtype" not in x] + [dict(dtype=0), dict(dtype=1), dict(dtype=2), dict(dtype=5),
                                 dict(dtype=-1), dict(scales=None), dict(scales=FAKE + 2)], ids=str)
def test_bad_caches_are_refused(bad):
    assert set(every_call(kv8(**bad), wide.batch()).values()) == {EINVAL}
    assert load_library().swift_coded_prefix_workspace_bytes(C.byref(kv8(**bad)), C.byref(wide.batch()), 4, 4, 1) == 0


@pytest.mark.parametrize("bad", wide.BAD_BATCHES, ids=str)
def test_bad_batches_are_refused(bad):
    assert set(every_call(kv8(), wide.batch(**bad)).values()) == {EINVAL}
    assert load_library().swift_coded_prefix_workspace_bytes(C.byref(kv8()), C.byref(wide.batch(**bad)), 4, 4, 1) == 0


def test_too_many_sequences_are_refused():
    assert set(every_call(kv8(), wide.batch(n_seqs=4097)).values()) == {ECAPACITY}


@pytest.mark.parametrize("bad", wide.BAD_ATTENTION, ids=str)
def test_bad_attention_arguments_are_refused(bad):
    got = every_call(kv8(), wide.batch(), a=wide.attention(**bad), x=append(block=9))
    assert got == {"append": EINVAL, "prompt": EINVAL, "prefix": EINVAL}
    assert load_library().swift_batch_error()


@pytest.mark.parametrize("bad", wide.BAD_APPEND, ids=str)
def test_bad_append_arguments_are_refused(bad):
    assert load_library().swift_coded_append(C.byref(kv8()), C.byref(wide.batch()), C.byref(append(**bad)), None) == EINVAL


def test_types_of_q_k_v_and_the_result():
    lib = load_library()
    for t in (-1, 3, 4):
        assert lib.swift_coded_append(C.byref(kv8()), C.byref(wide.batch()), C.byref(append(x_dtype=t)), None) == EUNSUPPORTED
        assert lib.swift_coded_prompt_attention(C.byref(kv8()), C.byref(wide.batch()), C.byref(wide.attention()), t, None) == EINVAL
        assert lib.swift_coded_prefix_workspace_bytes(C.byref(kv8()), C.byref(wide.batch()), 4, 4, t) == 0
    assert lib.swift_kv_append(C.byref(wide.kv(dtype=3)), C.byref(wide.batch()), C.byref(append()), None) == EINVAL


def test_null_structures_are_refused():
    lib = load_library()
    b, a = wide.batch(), wide.attention()
    assert lib.swift_coded_append(None, None, None, None) == EINVAL
    assert lib.swift_coded_append(C.byref(kv8()), C.byref(b), None, None) == EINVAL
    assert lib.swift_coded_prompt_attention(None, C.byref(b), C.byref(a), 1, None) == EINVAL
    assert lib.swift_coded_prompt_attention(C.byref(kv8()), C.byref(b), None, 1, None) == EINVAL
    assert lib.swift_coded_prefix_attention(C.byref(kv8()), None, C.byref(a), 1, 4, _DevBuf(FAKE, 1 << 40), None) == EINVAL


@pytest.mark.parametrize("x_dtype", [0, 1, 2])
@pytest.mark.parametrize("dim", [64, 128, 40, 256])
def test_workspaces_that_do_not_fit_are_refused(x_dtype, dim):
    lib = load_library()
    k, b = kv8(head_dim=dim), wide.batch(prefix_pages=FAKE, prefix_len=50)
    need = lib.swift_coded_prefix_workspace_bytes(C.byref(k), C.byref(b), 4, 4, x_dtype)
    assert need > 0
    a = wide.attention(q=paged._Rows(FAKE, 4 * dim, dim))
    call = lambda ws, rows=4: lib.swift_coded_prefix_attention(C.byref(k), C.byref(b), C.byref(a), x_dtype, rows, ws, None)
    assert call(_DevBuf(FAKE, need - 1)) == ECAPACITY
    assert call(_DevBuf(None, need)) == EINVAL
    assert call(_DevBuf(FAKE + 16, need)) == EINVAL
    assert call(_DevBuf(FAKE, need), rows=0) == EINVAL
    assert lib.swift_coded_prefix_workspace_bytes(C.byref(k), C.byref(b), 3, 4, x_dtype) == 0
    assert lib.swift_coded_prefix_workspace_bytes(C.byref(k), C.byref(b), 4, 0, x_dtype) == 0


def test_empty_batches_do_nothing():
    assert set(every_call(kv8(), wide.batch(n_seqs=0, row_start=None, kv_len=None, page_table=None)).values()) == {0}
    assert set(every_call(kv8(), wide.batch(n_rows=0)).values()) == {0}


def test_host_tensors_are_refused():
    with pytest.raises(ValueError, match="CUDA"):
        paged.PagedKV(torch.zeros(2, 1, 2, 1, 8, 64, dtype=torch.int8), torch.zeros(2, 1, 2, 1))
    with pytest.raises(ValueError, match="CUDA"):
        sampling.sample_rows(torch.zeros(2, 8), torch.zeros(2))


# ----------------------------------------------------------------------------------------------- sample_rows
def sample(**kw):
    v = dict(n_rows=2, vocab=1000, dtype=0, logits=FAKE, row_stride=1000, uniforms=FAKE, temperature=None, temperature_all=1.0, top_k=None,
             top_k_all=0, top_p=None, top_p_all=1.0, min_p=None, min_p_all=0.0, tokens=FAKE, probs=FAKE)
    v.update(kw)
    return sampling._Sample(**v)


@pytest.mark.parametrize("bad", [dict(n_rows=-1), dict(n_rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=262145), dict(dtype=3), dict(dtype=-1), dict(logits=None),
                                 dict(logits=FAKE + 2), dict(logits=FAKE + 1, dtype=1), dict(row_stride=-1), dict(uniforms=None), dict(uniforms=FAKE + 2),
                                 dict(temperature=FAKE + 1), dict(top_k=FAKE + 2), dict(top_p=FAKE + 3), dict(min_p=FAKE + 1), dict(tokens=None),
                                 dict(tokens=FAKE + 2), dict(probs=FAKE + 2)], ids=str)
def test_bad_sample_arguments_are_refused(bad):
    assert load_library().swift_sample_rows(C.byref(sample(**bad)), None) == EINVAL
    assert load_library().swift_batch_error()


def test_no_rows_are_no_work():
    assert load_library().swift_sample_rows(C.byref(sample(n_rows=0, logits=None, uniforms=None, tokens=None)), None) == 0
    assert load_library().swift_sample_rows(None, None) == EINVAL
