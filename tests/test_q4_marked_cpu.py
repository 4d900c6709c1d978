"""A cache marked as held in 4 bits: the calls that take its pools for rows of values refuse it on the host."""
import ctypes

import pytest

from paper_2609_03515_gb300 import DecodeCache, Q4Cache, ikv

A = 64  # an address on a 16-byte boundary, never read
BIG = ctypes.c_size_t(1 << 40)


def structs(bits):
    s = ikv.ikv_shape(batch=2, layers=3, q_heads=8, kv_heads=2, head_dim=64, dtype=ikv.IKV_BF16, granularity=ikv.IKV_GRAN_SEQ)
    c = ikv.ikv_cache(k=A, v=A, block_table=A, num_pages=9, page_size=16, max_pages=4, len=A, pos=A, next_pos=A, max_len=60,
                      start=A, vnorm=A, code_bits=bits)
    p = ikv.ikv_params(alpha=0.5, refresh_period=1, budget=A)
    return ctypes.byref(s), ctypes.byref(c), ctypes.byref(p)


def dense_calls(bits):
    s, c, p = structs(bits)
    n = ctypes.byref(ikv.SZ(0))
    half = ctypes.c_float(0.5)
    return {
        "ikv_decode_attend_score": (s, c, 0, A, A, A, None, half, A, BIG, None),
        "ikv_value_norms": (s, c, None),
        "ikv_compact_workspace_size": (s, c, ikv.IKV_COMPACT_STABLE, n),
        "ikv_compact_kv": (s, c, A, A, None, ikv.IKV_COMPACT_STABLE, A, BIG, None),
        "ikv_append_token": (s, c, A, A, None, 0, A, BIG, None),
        "ikv_step_workspace_size": (s, c, n),
        "ikv_step": (s, p, c, A, 1, A, A, A, A, A, BIG, None),
        "ikv_step_begin": (s, p, c, A, 1, A, BIG, None),
        "ikv_step_layer": (s, p, c, A, 1, 0, A, A, A, A, A, BIG, None),
        "ikv_step_end": (s, p, c, A, 1, A, BIG, None),
    }


@pytest.mark.parametrize("name", list(dense_calls(0)))
def test_dense_calls_refuse_it(name):
    n = ikv.ikv_launch_count()
    assert ikv.raw_status(name, *dense_calls(4)[name]) == ikv.IKV_ERR_UNSUPPORTED and "4 bits" in ikv.ikv_last_error()
    assert ikv.raw_status(name, *dense_calls(3)[name]) == ikv.IKV_ERR_ARG
    assert ikv.ikv_launch_count() == n


@pytest.mark.parametrize("bits", [0, 4])
def test_the_others_take_it(bits):
    """Up to the check that each call fails next."""
    s, c, _ = structs(bits)
    q4 = ctypes.byref(ikv.ikv_q4(A, A))
    rows = ctypes.byref(ikv.ikv_rows(1024, 512, 128, 64, None))
    assert ikv.raw_status("ikv_q4_store", s, c, q4, 0, 1, None, A, rows, None, None, 1, None) == ikv.IKV_ERR_ARG
    assert ikv.raw_status("ikv_q4_append_token", s, c, q4, A, A, None, 0, None, None) == ikv.IKV_ERR_ARG
    assert ikv.raw_status("ikv_q4_attend_score", s, c, q4, 0, A, A, None, None, ctypes.c_float(0), None, BIG, None) == ikv.IKV_ERR_WORKSPACE
    assert ikv.raw_status("ikv_attend_workspace_size", s, c, ctypes.byref(ikv.SZ(0))) == ikv.IKV_OK
    assert ikv.raw_status("ikv_pages_workspace_size", s, c, None, None) == ikv.IKV_ERR_ARG


def test_the_classes_mark_theirs():
    q = Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16)
    d = DecodeCache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16)
    assert q.cache().code_bits == 4 and d.cache().code_bits == 0
    with pytest.raises(ikv.IKVError):
        q.step_workspace()
    assert d.step_workspace().numel() > 0
