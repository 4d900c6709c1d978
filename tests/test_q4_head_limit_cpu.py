"""More query heads than the 4-bit attention's score pass holds."""
import ctypes

import pytest

from paper_2609_03515_gb300 import ikv

A = 64  # an address on a 16-byte boundary, never read


@pytest.mark.parametrize("kv_heads,want", [(1025, ikv.IKV_ERR_SHAPE), (1024, ikv.IKV_ERR_WORKSPACE)])
def test_query_heads(kv_heads, want):
    s = ikv.ikv_shape(batch=1, layers=1, q_heads=8 * kv_heads, kv_heads=kv_heads, head_dim=64, dtype=ikv.IKV_BF16,
                      granularity=ikv.IKV_GRAN_SEQ)
    c = ikv.ikv_cache(k=A, v=A, block_table=A, num_pages=9, page_size=16, max_pages=4, len=A, pos=A, next_pos=A, max_len=60)
    st = ikv.raw_status("ikv_q4_attend_score", ctypes.byref(s), ctypes.byref(c), ctypes.byref(ikv.ikv_q4(A, A)), 0, A, A, None,
                        None, ctypes.c_float(0), None, ctypes.c_size_t(0), None)
    assert st == want  # (what is allowed fails at its workspace, which is not given)
