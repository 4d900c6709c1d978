"""Values that are not finite where single rows of a unit do not look: those rows are computed again over what they see,
however long that is, and every other row keeps its bits."""
import math

import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import DT, Cache, attention, window_seen
from test_gpu_prefix import Call, reference

pytestmark = pytest.mark.gpu


class Window:
    def __init__(self, c, count, window, sinks):
        self.c = c
        self.q = torch.randn(count, c.h * c.d, generator=torch.Generator().manual_seed(8)).to(DT[c.dtype])
        self.qd, self.out = self.q.cuda(), torch.empty(count, c.h * c.d, dtype=DT[c.dtype], device="cuda")
        self.n = torch.tensor([count], dtype=torch.int32).cuda()
        self.win = ikv.ikv_window(window, sinks, None, self.n.data_ptr(), count, 0, 0)
        self.ws = torch.empty(ikv.ikv_window_workspace_size(c.shape(), c.cache(), self.win), dtype=torch.uint8,
                              device="cuda")

    def run(self):
        self.out.fill_(77.0)
        ikv.ikv_window_attend(self.c.shape(), self.c.cache(), self.win, 0, self.qd, self.out, self.ws, self.ws.numel())
        torch.cuda.synchronize()
        assert ikv.ikv_device_status() == 0
        return self.out.clone()

    def close(self, out, rows, window, sinks, cols=slice(None)):
        """Rows of `out` against 64 bits, over the cache as its host copy is."""
        c, count = self.c, self.q.shape[0]
        n = c.lens[0]
        for h in range(c.h):
            for i in rows:
                seen = window_seen(n, count, i, i + 1, window, sinks)
                at = slice(h * c.d, (h + 1) * c.d)
                ref, _, tol, _ = attention(c, 0, 0, h // c.G, self.q[i:i + 1, at], seen)
                worst = ((out[i, at].cpu().double() - ref[0]).abs() / tol[0])[cols].nan_to_num(nan=math.inf).amax().item()
                assert worst <= 1.0, (h, i, worst)


def near(a, b, c):
    """Two evaluations of the same outputs: each rounds its weights (half a step of bf16, 2^-8 of sum p |V| at most, in
    all) and its result, 2^-8 again; sum p |V| is at most the largest |V|.  4 * 2^-8 of that, and 2^-12 for what 32
    bits leave (3000 terms or parts, 2^-24 each)."""
    return bool(((a.float() - b.float()).abs() <= (2.0 ** -6 + 2.0 ** -12) * c.v[0].abs().amax().item()).all())


def put(c, which, slot, channel, value):
    at = slot + c.starts[0]
    pool = c.t[which]
    pool[0, int(c.table[0][at // c.page]), :, at % c.page, channel] = value


@pytest.mark.parametrize("bad", [10, 100000])
def test_a_long_prompt_with_an_infinite_value(bad):
    """128k tokens, every earlier slot visible: a part has up to 1024 tiles and 256 rows, and the rows of the slot's own
    unit in front of it are the ones to be computed again."""
    n = 131072
    c = Cache([n], 1, 1, 64, "bf16", 64, seed=30, layers=1).device(9.0)
    w = Window(c, n, 0, 0)
    clean = w.run()
    put(c, "v", bad, 5, math.inf)
    out = w.run()
    assert bool((out[bad:, 5] == math.inf).all())
    rest = [i for i in range(c.d) if i != 5]
    assert torch.equal(out[bad:, rest], clean[bad:, rest])  # (they see it: nothing is wrong with them)
    first = bad // 256 * 256
    assert torch.equal(out[:first], clean[:first])
    assert bool(out[first:bad].isfinite().all())
    w.close(out, sorted({first, bad // 2, bad - 1}), 0, 0) if bad < 256 else w.close(out, [first, bad - 1], 0, 0)
    assert near(out[first:bad], clean[first:bad], c)


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("bf16", 16), ("f32", 16)])
@pytest.mark.parametrize("group,window,sinks", [(1, 0, 0), (8, 0, 0), (4, 700, 4), (7, 129, 130)])
@pytest.mark.parametrize("which,value", [("v", math.inf), ("v", math.nan), ("k", math.nan)])
def test_prompts_of_many_parts(dtype, page, group, window, sinks, which, value):
    """Several bad tokens over 3000, and shares of several parts, cut pairs among them."""
    n, d = 3000, 64
    c = Cache([n], 4, group, d, dtype, page, seed=31, layers=1, starts=[11]).device(9.0)
    w = Window(c, n, window, sinks)
    clean = w.run()
    bad = [0, 517, 518, 2047, 2999] if which == "v" else [1500]
    for s in bad:
        put(c, which, s, 7, value)
    out = w.run().view(n, c.h, d)
    clean = clean.view(n, c.h, d)
    p, j = torch.arange(n)[:, None], torch.tensor(bad)[None]
    sees = ((j <= p) & ((j > p - window) | (window == 0) | (j < sinks))).any(1).cuda()
    hit = out[sees]
    if which == "k":
        assert bool(hit.isnan().all())
    else:
        rest = [i for i in range(d) if i != 7]
        assert bool((hit[..., 7].isnan() if math.isnan(value) else (hit[..., 7] == value)).all())
        assert near(hit[..., rest], clean[sees][..., rest], c)
    free = out[~sees]
    assert bool(free.isfinite().all())
    assert near(free, clean[~sees], c)
    hidden = (~sees).nonzero().flatten().tolist()
    w.close(out.view(n, -1), hidden[::max(1, len(hidden) // 20)], window, sinks)


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("members", [3, 40])
def test_a_prefix_whose_dead_rows_are_not_finite(dtype, page, members):
    """Dead rows hold NaN and infinities; single members see some of them.  Scores of the others stay exact."""
    lens = [4000 + i for i in range(members)]
    share = [(0, list(range(1, members)), 3990)]
    c = Cache(lens, 2, 4, 64, dtype, page, seed=32, layers=1, share=share, dead=0.2).device(9.0)
    clean = Cache(lens, 2, 4, 64, dtype, page, seed=32, layers=1, share=share, dead=0.2)
    nobody, one, both = 100, 2500, 3600
    for x in (c, clean):
        x.pos[:, nobody] = x.pos[:, one] = -1
        x.pos[1, one] = one
        x.pos[:, both] = -1
        x.pos[0, both] = x.pos[2, both] = both
    c.t["pos"].copy_(c.pos)
    for s in (nobody, one):
        put(c, "v", s, 3, math.nan)
    put(c, "v", both, 9, -math.inf)
    put(c, "k", nobody, 0, math.nan)
    call = Call(c, [list(range(members))], [3990], layer=0, ema=True)
    call.run()
    call.done()
    got, score = call.out.cpu().double(), call.score.cpu().double()
    call.c = clean
    out, tol, want, stol = reference(call)
    bad = torch.zeros(members, c.h, 64, dtype=torch.bool)
    bad[1, :, 3] = True
    bad[0, :, 9] = bad[2, :, 9] = True
    assert bool(got[1, :, 3].isnan().all())
    assert bool((got[[0, 2]][:, :, 9] == -math.inf).all())
    assert bool(((got - out).abs() <= tol)[~bad].all())
    for b, n in enumerate(lens):
        assert bool(((score[b, :n] - want[b, :n]).abs() <= stol[b, :n]).all())
