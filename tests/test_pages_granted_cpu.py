"""Calls that do not go by what ikv_pages_writable granted refuse a cache that does, on the host."""
import ctypes

import pytest

from paper_2609_03515_gb300 import DecodeCache, Q4Cache, ikv

A = 64  # an address on a 16-byte boundary, never read
BIG = ctypes.c_size_t(1 << 40)


def structs(writable):
    s = ikv.ikv_shape(batch=2, layers=3, q_heads=8, kv_heads=2, head_dim=64, dtype=ikv.IKV_BF16, granularity=ikv.IKV_GRAN_SEQ)
    c = ikv.ikv_cache(k=A, v=A, block_table=A, num_pages=9, page_size=16, max_pages=4, len=A, pos=A, next_pos=A, max_len=60,
                      start=A, writable=writable)
    return ctypes.byref(s), ctypes.byref(c), ctypes.byref(ikv.ikv_params(alpha=0.5, refresh_period=1, budget=A))


@pytest.mark.parametrize("name", ["ikv_compact_kv", "ikv_step", "ikv_step_begin", "ikv_step_layer", "ikv_step_end"])
def test_steps_and_compactions_in_place(name):
    s, c, p = structs(A)
    args = {
        "ikv_compact_kv": (s, c, A, A, None, ikv.IKV_COMPACT_STABLE, A, BIG, None),
        "ikv_step": (s, p, c, A, 1, A, A, A, A, A, BIG, None),
        "ikv_step_begin": (s, p, c, A, 1, A, BIG, None),
        "ikv_step_layer": (s, p, c, A, 1, 0, A, A, A, A, A, BIG, None),
        "ikv_step_end": (s, p, c, A, 1, A, BIG, None),
    }[name]
    n = ikv.ikv_launch_count()
    assert ikv.raw_status(name, *args) == ikv.IKV_ERR_UNSUPPORTED and ikv.ikv_launch_count() == n


def test_page_calls_want_it_aligned():
    s, c, _ = structs(A + 4)
    p = ikv.ikv_pages()
    p.refs, p.n_planes, p.plane[0], p.row_bytes[0] = A, 1, A, 128
    assert ikv.raw_status("ikv_pages_release", s, c, ctypes.byref(p), 0, None) == ikv.IKV_ERR_ALIGN


def test_what_the_classes_give():
    q = Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16, pool_pages=5)
    d = DecodeCache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16, pool_pages=5)
    assert q.cache().writable == q.writable.data_ptr() and q.cache(granted=False).writable is None
    assert d.cache().writable is None and d.cache(granted=True).writable == d.writable.data_ptr()
    assert Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16).cache().writable is None
