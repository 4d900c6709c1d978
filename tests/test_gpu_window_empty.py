"""ikv_window_attend where whole units of queries see no slot, beside units that see many: their rows are zeros,
every other row is its own sequence's, call after call."""
import math

import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import DT, MARK, Cache, attention, window_seen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,page", [("f32", 16), ("bf16", 20), ("bf16", 16)])
@pytest.mark.parametrize("group,d", [(1, 128), (8, 64), (7, 64)])
def test_units_without_a_slot_between_full_ones(dtype, page, group, d):
    """Empty sequences, and ones with more queries than slots, so that units of 64 rows lie wholly in front of the
    first slot.  A CTA meets such units behind full ones and behind units of few rows, some as its first."""
    torch.manual_seed(1)
    lens, counts = [], []
    for i in range(90):
        n, c = [(150, 70), (0, 64), (33, 1), (0, 1), (5, 140), (0, 9), (40, 40), (2, 65), (0, 130)][i % 9]
        lens.append(n)
        counts.append(c)
    cache = Cache(lens, 2, group, d, dtype, page, seed=1, layers=1).device()
    width = cache.h * d
    row0 = [sum(counts[:b]) for b in range(len(counts))]
    rows = sum(counts)
    q = torch.randn(rows, width).to(DT[dtype])
    qd, out = q.cuda(), torch.empty(rows + 64, width, dtype=DT[dtype], device="cuda")
    r0, cn = torch.tensor(row0, dtype=torch.int32).cuda(), torch.tensor(counts, dtype=torch.int32).cuda()
    win = ikv.ikv_window(50, 3, r0.data_ptr(), cn.data_ptr(), max(counts), 0, 0)
    shape, pools = cache.shape(), cache.cache()
    n = ikv.ikv_window_workspace_size(shape, pools, win)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def call():
        out.fill_(MARK)
        ikv.ikv_window_attend(shape, pools, win, 0, qd, out, ws, n)

    call()
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 0
    got = out.cpu()
    assert bool((got[rows:] == MARK).all())
    for b, (m, c) in enumerate(zip(lens, counts)):
        hidden = max(0, c - m)
        assert bool((got[row0[b]:row0[b] + hidden] == 0).all()), b
        if m == 0:
            continue
        seen = window_seen(m, c, hidden, c, 50, 3)
        for h in range(cache.h):
            cols = slice(h * d, (h + 1) * d)
            at = slice(row0[b] + hidden, row0[b] + c)
            ref, _, tol, _ = attention(cache, 0, b, h // group, q[at, cols], seen)
            worst = ((got[at, cols].double() - ref).abs() / tol).nan_to_num(nan=math.inf).amax().item()
            assert worst <= 1.0, (b, h, worst)
    first = out.clone()
    for i in range(300):
        call()
        assert torch.equal(out, first), i
    assert ikv.ikv_device_status() == 0
