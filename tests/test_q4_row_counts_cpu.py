"""Rows that 32 bits just hold: the kernels of the 4-bit store and load count up to a CTA's rows past them."""
import ctypes

import pytest

from paper_2609_03515_gb300 import ikv

A = 64  # an address on a 16-byte boundary, never read


@pytest.mark.parametrize("name", ["ikv_q4_store", "ikv_q4_load"])
@pytest.mark.parametrize("kv_heads,most", [(2, (1 << 30) - 1), (4, 1 << 29), (16, (1 << 27) - 1), (16, (1 << 27) - 4095), (3, 0x2aaaaaaa)])
def test_too_many_rows_are_refused(name, kv_heads, most):
    s = ikv.ikv_shape(batch=1, layers=1, q_heads=kv_heads, kv_heads=kv_heads, head_dim=64, dtype=ikv.IKV_BF16,
                      granularity=ikv.IKV_GRAN_SEQ)
    c = ikv.ikv_cache(k=A, v=A, block_table=A, num_pages=9, page_size=16, max_pages=1 << 26, len=A, pos=A, next_pos=A, max_len=0)
    st = ikv.raw_status(name, ctypes.byref(s), ctypes.byref(c), ctypes.byref(ikv.ikv_q4(A, A)), 0, 1, A, A,
                        ctypes.byref(ikv.ikv_rows(1024, 512, 128, 64, None)), None, None, most, None)
    assert st == ikv.IKV_ERR_SHAPE and "max_count * kv_heads" in ikv.ikv_last_error()
