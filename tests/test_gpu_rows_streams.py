"""Calls at once: shared-prefix, window and plain decode attention on streams of their own, with workspaces of their own,
give what they give alone."""
import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import DT, MARK, Cache
from test_gpu_prefix import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_two_kinds_of_calls_on_three_streams(dtype, d):
    lens = [900, 880, 950, 1200, 40]
    c = Cache(lens, 4, 4, d, dtype, 64, seed=51, share=[(0, [1, 2], 870)]).device(9.0)
    prefix = Call(c, [[0, 1, 2]], [870], score=True)
    counts = [300, 1, 950, 17, 40]
    row0 = [sum(counts[:b]) for b in range(len(counts))]
    q = torch.randn(sum(counts), c.h * d, generator=torch.Generator().manual_seed(9)).to(DT[dtype]).cuda()
    out = torch.empty_like(q)
    r0, cn = [torch.tensor(x, dtype=torch.int32).cuda() for x in (row0, counts)]
    win = ikv.ikv_window(200, 4, r0.data_ptr(), cn.data_ptr(), max(counts), 0, 0)
    shape, cache = c.shape(), c.cache()
    n = ikv.ikv_window_workspace_size(shape, cache, win)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dout, dscore = torch.empty_like(prefix.out), torch.empty_like(prefix.score)
    dn = ikv.ikv_attend_workspace_size(shape, cache)
    dws = torch.empty(dn, dtype=torch.uint8, device="cuda")
    calls = [prefix.run, lambda st: ikv.ikv_window_attend(shape, cache, win, 1, q, out, ws, n, st),
             lambda st: ikv.ikv_decode_attend_score(shape, cache, 1, prefix.qd, dout, dscore, None, 0.0, dws, dn, st)]
    kept = [prefix.out, prefix.score, out, dout, dscore]

    def mark():
        for x in kept:
            x.fill_(MARK)
        torch.cuda.synchronize()

    mark()
    for f in calls:
        f(torch.cuda.current_stream())
        torch.cuda.synchronize()
    alone = [x.clone() for x in kept]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        mark()
        for _ in range(20):
            for f, st in zip(calls, streams):
                f(st)
        torch.cuda.synchronize()
        for a, b in zip(kept, alone):
            assert torch.equal(a, b)
    assert ikv.ikv_device_status() == 0
