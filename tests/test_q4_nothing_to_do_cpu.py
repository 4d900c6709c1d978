"""Stores and loads of no rows or no layers: done at once, and nothing is launched.  Each call runs in a
process of its own, so that one that ends its process fails its test alone."""
import subprocess
import sys

import pytest

CALL = """
import ctypes
from paper_2609_03515_gb300 import ikv
A = 64  # an address on a 16-byte boundary, never read
s = ikv.ikv_shape(batch=2, layers=3, q_heads=8, kv_heads=2, head_dim=%d, dtype=%d, granularity=ikv.IKV_GRAN_SEQ)
c = ikv.ikv_cache(k=A, v=A, block_table=A, num_pages=9, page_size=16, max_pages=4, len=A, pos=A, next_pos=A, max_len=60)
r = ikv.ikv_rows(layer=1024, seq=512, token=128, head=64, row0=None)
n = ikv.ikv_launch_count()
ikv.%s(s, c, ikv.ikv_q4(A, A), 0, %d, A, A, r, None, None, %d, 0)
assert ikv.ikv_launch_count() == n
print("done")
"""


@pytest.mark.parametrize("name", ["ikv_q4_store", "ikv_q4_load"])
@pytest.mark.parametrize("layers,most", [(1, 0), (0, 5), (0, 0), (3, 0)])
@pytest.mark.parametrize("d,dtype", [(64, 0), (128, 1)])
def test_no_rows(name, layers, most, d, dtype):
    r = subprocess.run([sys.executable, "-c", CALL % (d, dtype, name, layers, most)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "done", (r.returncode, r.stderr[-300:])
