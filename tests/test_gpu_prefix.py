"""ikv_prefix_attend_score against a 64-bit evaluation: groups of any size, prefixes that end anywhere, members
whose own pages hold something else there, dead slots of each member, wrong member lists."""
import math

import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import DT, MARK, Cache, attention

pytestmark = pytest.mark.gpu


def lists(groups):
    first = [0]
    for m in groups:
        first.append(first[-1] + len(m))
    return first, [b for m in groups for b in m]


class Call:
    def __init__(self, c, groups, plens, layer=1, score=True, ema=False, alpha=0.75, seed=5, first=None, member=None):
        self.c, self.layer, self.alpha = c, layer, alpha
        nb, h, d = len(c.lens), c.h, c.d
        f, m = lists(groups)
        self.q = torch.randn(nb, h, d, generator=torch.Generator().manual_seed(seed)).to(DT[c.dtype])
        self.qd = self.q.cuda()
        self.out = torch.full((nb, h, d), MARK, dtype=DT[c.dtype], device="cuda")
        rows = c.pos.shape[0]
        self.score = torch.full((rows, c.cap), MARK, device="cuda") if score else None
        self.ema0 = torch.rand(rows, c.cap, generator=torch.Generator().manual_seed(6))
        self.ema = self.ema0.cuda() if ema else None
        self.dev = [torch.tensor(x, dtype=torch.int32).cuda() for x in (first or f, member or m, plens)]
        self.prefix = ikv.ikv_prefix(len(plens), *[x.data_ptr() for x in self.dev])
        self.shape, self.cache = c.shape(), c.cache()
        self.n = ikv.ikv_prefix_workspace_size(self.shape, self.cache, self.prefix)
        self.ws = torch.full((self.n + 256,), 0xA5, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        ikv.ikv_prefix_attend_score(self.shape, self.cache, self.prefix, self.layer, self.qd, self.out, self.score,
                                    self.ema, self.alpha, self.ws, self.n, stream or torch.cuda.current_stream())

    def done(self, status=0):
        torch.cuda.synchronize()
        assert ikv.ikv_device_status() == status
        assert bool((self.ws[self.n:] == 0xA5).all())


def reference(call):
    c = call.c
    nb = len(c.lens)
    per = c.g if c.gran == "kvhead" else 1
    out = torch.zeros(nb, c.h, c.d, dtype=torch.float64)
    tol = torch.zeros_like(out)
    score = torch.zeros(nb * per, c.cap, dtype=torch.float64)
    stol = torch.zeros_like(score)
    for b, n in enumerate(c.lens):
        if n == 0:
            continue
        for i in range(c.g):
            seen = (c.alive(b, i) if c.dead else torch.ones(n, dtype=torch.bool))[None].expand(c.G, n)
            hs = slice(i * c.G, (i + 1) * c.G)
            out[b, hs], p, tol[b, hs], pt = attention(c, call.layer, b, i, call.q[b, hs], seen)
            r = b * per + (i if per > 1 else 0)
            score[r, :n] += p.sum(0) / (c.G if per > 1 else c.h)
            stol[r, :n] += pt.sum(0) / (c.G if per > 1 else c.h)
    return out, tol, score, stol + 1e-30


def check(c, groups, plens, status=0, **kw):
    call = Call(c, groups, plens, **kw)
    call.run()
    call.done(status)
    out, tol, score, stol = reference(call)
    err = ((call.out.cpu().double() - out).abs() / (tol + 1e-30)).nan_to_num(nan=math.inf)
    assert err.amax().item() <= 1.0, (err.amax().item(), err.flatten(1).amax(1))
    per = c.g if c.gran == "kvhead" else 1
    inside = torch.arange(c.cap)[None] < torch.tensor(c.lens).repeat_interleave(per)[:, None]
    if call.score is not None:
        got = call.score.cpu().double()
        assert bool((got[~inside] == MARK).all())
        assert bool(((got - score).abs() <= stol)[inside].all())
    if call.ema is not None:
        # two products and a sum in 32 bits, one of them perhaps with the product unrounded
        want = call.alpha * call.ema0.double() + (1 - call.alpha) * score
        got = call.ema.cpu().double()
        assert bool((got[~inside] == call.ema0.double()[~inside]).all())
        assert bool(((got - want).abs() <= stol + 4 * 2.0 ** -24 * want.abs() + 1e-30)[inside].all())
    return call


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("bf16", 20), ("f32", 16)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 7, 8])
@pytest.mark.parametrize("gran,hidden", [("seq", math.nan), ("kvhead", math.nan), ("seq", 9.0)])
def test_shapes(dtype, page, d, group, gran, hidden):
    lens = [200, 180, 131, 150, 133, 1, 77]
    c = Cache(lens, 2, group, d, dtype, page, seed=1, gran=gran, share=[(0, [3, 1], 130), (4, [2], 129)]).device(hidden)
    check(c, [[0, 3, 1], [4, 2]], [130, 129], ema=True)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 24), ("bf16", 5), ("f32", 16)])
@pytest.mark.parametrize("plen", [0, 1, 127, 128, 129, 255, 256, 300])
@pytest.mark.parametrize("start", [0, 9, 128])
@pytest.mark.parametrize("hidden", [math.nan, 9.0])
def test_prefixes_end_anywhere(dtype, page, plen, start, hidden):
    lens = [300, 301, 300, 420]
    c = Cache(lens, 1, 4, 128, dtype, page, seed=2, starts=[start] * 4, share=[(1, [0, 2, 3], plen)]).device(hidden)
    check(c, [[1, 0, 3, 2]], [plen])
    check(c, [[1, 0, 3, 2]], [plen], layer=0, score=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prefix_longer_than_a_member_is_cut(dtype):
    lens = [300, 90, 200, 0]
    c = Cache(lens, 2, 2, 64, dtype, 16, seed=3, share=[(0, [1], 90), (0, [2], 90)]).device()
    check(c, [[0, 1, 2]], [250], ema=True)
    check(c, [[0, 1, 2, 3]], [250])  # (an empty member leaves nothing to share)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4, 7])
@pytest.mark.parametrize("members", [2, 18, 19, 40, 150])
def test_group_sizes(dtype, group, members):
    """Rows that fill one tile of 128, go beyond it, fill two, go beyond those."""
    lens = [190 + i % 5 for i in range(members)] + [40, 7]
    order = [(i * 7) % members for i in range(members)] if members % 7 else list(range(members))
    c = Cache(lens, 1, group, 64 if members > 100 else 128, dtype, 16, seed=4, layers=2,
              share=[(order[0], order[1:], 188)]).device(9.0)
    check(c, [order], [188], score=members < 50)


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("bf16", 12), ("f32", 16)])
@pytest.mark.parametrize("gran", ["seq", "kvhead"])
@pytest.mark.parametrize("dead", [0.2, 0.95, 1.0])
@pytest.mark.parametrize("hidden", [math.nan, 9.0])
def test_dead_slots_are_each_members_own(dtype, page, gran, dead, hidden):
    lens = [200, 260, 240, 300, 50]
    c = Cache(lens, 2, 4, 128, dtype, page, seed=5, dead=dead, gran=gran, starts=[0, 5, 0, 0, 70],
              share=[(1, [0, 2], 170)]).device(hidden)
    check(c, [[1, 0, 2]], [170], ema=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_only_the_first_members_prefix_is_read(dtype):
    """The other members' slots of the prefix hold NaN in their own pages, and need no page of their own."""
    lens = [150, 160, 170]
    c = Cache(lens, 2, 4, 128, dtype, 16, seed=6, share=[(0, [1, 2], 128)])
    keep = [x.clone() for x in c.k], [x.clone() for x in c.v]
    for b in (1, 2):
        c.k[b][:, :, :128] = math.nan
        c.v[b][:, :, :128] = math.nan
    c.device()
    c.k, c.v = keep
    check(c, [[0, 1, 2]], [128], ema=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_dead_row_that_is_not_finite_reaches_only_the_members_that_see_it(dtype):
    lens = [150, 160, 170]
    c = Cache(lens, 1, 2, 128, dtype, 16, seed=7, share=[(0, [1, 2], 128)])
    clean = Cache(lens, 1, 2, 128, dtype, 16, seed=7, share=[(0, [1, 2], 128)])
    for b in range(3):
        c.k[b][:, :, 60] = math.nan
        c.v[b][:, :, 60] = -math.inf
    c.dead = clean.dead = 1e-9
    for x in (c, clean):
        x.pos[0, 60] = x.pos[2, 60] = -1  # sequence 1 sees it
    call = Call(c.device(), [[0, 1, 2]], [128])
    call.run()
    call.done()
    call.c = clean
    out, tol, score, stol = reference(call)
    got = call.out.cpu().double()
    assert bool(got[1].isnan().all())
    for b in (0, 2):
        assert bool(((got[b] - out[b]).abs() <= tol[b]).all())
        n = lens[b]
        assert bool(((call.score[b, :n].cpu().double() - score[b, :n]).abs() <= stol[b, :n]).all())
    assert bool(call.score[1, :160].isnan().all())


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 24), ("f32", 16)])
def test_a_prefix_up_to_the_first_members_end(dtype, page):
    """Nothing of the first member's own, NaN behind it; a slot space that is full."""
    lens = [5 * page - 7, 5 * page - 7 + 1, 5 * page]
    c = Cache(lens, 2, 4, 128, dtype, page, seed=14, share=[(0, [1, 2], lens[0])], extra_pages=0).device()
    check(c, [[0, 1, 2]], [lens[0]], ema=True)
    check(c, [[0, 1, 2]], [5 * page])


def test_no_groups_and_lone_members():
    lens = [130, 61, 300]
    c = Cache(lens, 2, 4, 128, "bf16", 64, seed=8).device()
    check(c, [], [])
    check(c, [[1], [2]], [40, 40])
    one = Cache([5], 1, 1, 64, "f32", 16, seed=8).device()
    check(one, [], [])


def test_wrong_member_lists_are_reported_and_left_out():
    """A sequence named twice counts once, numbers out of range and entries behind the batch's are left out."""
    lens = [150, 150, 150, 90]
    c = Cache(lens, 2, 4, 128, "bf16", 16, seed=9, share=[(0, [1, 2], 140)]).device()
    check(c, [], [140], status=128, first=[0, 4], member=[0, 1, 1, 2])
    check(c, [], [140], status=128, first=[0, 4], member=[-1, 0, 4, 2])
    check(c, [], [140, 140], status=128, first=[0, 2, 4], member=[0, 1, 2, 0])
    check(c, [], [140], status=128, first=[0, 6], member=[0, 1, 2, 2, 1, 0])
    check(c, [], [140], status=128, first=[0, 6], member=[2, 2, 2, 2, 1, 0])
    # ranges that overlap: no group is used
    check(c, [], [140, 140, 140], status=128, first=[0, 3, 1, 3], member=[0, 1, 2])
    check(c, [], [140], status=128, first=[-1, 2], member=[0, 1])
    # a first entry behind 0 is no mistake
    check(c, [], [140], first=[1, 3], member=[99, 0, 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_prefix_split_over_the_gpu(dtype):
    lens = [9000 + 3 * i for i in range(5)] + [11000]
    c = Cache(lens, 2, 4, 128, dtype, 64, seed=10, layers=1, share=[(0, [1, 2, 3, 4], 9000)]).device()
    check(c, [[0, 1, 2, 3, 4]], [8999], layer=0)


def test_many_groups():
    """More groups and sequences than threads of a CTA."""
    n = 1100
    lens = [20 + i % 9 for i in range(2 * n)]
    c = Cache(lens, 1, 1, 64, "bf16", 8, seed=11, layers=1, share=[(i, [i + n], 18) for i in range(n)]).device(9.0)
    check(c, [[i, i + n] for i in range(n)], [18] * n, layer=0)


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("f32", 64)])
def test_like_the_plain_decode_call(dtype, page):
    """The same results as ikv_decode_attend_score, which reads the prefix once a sequence."""
    lens = [700, 650, 720]
    c = Cache(lens, 2, 4, 128, dtype, page, seed=12, share=[(0, [1, 2], 640)]).device(hidden=0.0)
    call = check(c, [[0, 1, 2]], [640], ema=True)
    out, score, ema = torch.zeros_like(call.out), torch.zeros_like(call.score), call.ema0.cuda()
    n = ikv.ikv_attend_workspace_size(call.shape, call.cache)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    ikv.ikv_decode_attend_score(call.shape, call.cache, 1, call.qd, out, score, ema, call.alpha, ws, n)
    torch.cuda.synchronize()
    _, tol, _, stol = reference(call)
    assert bool(((out.double() - call.out.double()).abs() <= 2 * tol.cuda()).all())
    for b, x in enumerate(lens):
        assert bool(((score[b, :x] - call.score[b, :x]).abs() <= 2 * stol[b, :x].cuda()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replayed_from_a_graph_with_lengths_that_grew(dtype):
    """A captured call reads lengths and groups from the device: the next steps' are the replay's."""
    lens = [900, 910, 905, 333]
    c = Cache(lens, 2, 4, 128, dtype, 64, seed=13, share=[(0, [1, 2], 890)]).device()
    call = Call(c, [[0, 1, 2]], [890])
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        call.run(st)
        st.synchronize()
        with torch.cuda.graph(g, stream=st):
            call.run(torch.cuda.current_stream())
    g.replay()
    call.done()
    first = call.out.clone(), call.score.clone()
    short = [880, 700, 905, 1]
    c.t["len"].copy_(torch.tensor(short, dtype=torch.int32))
    call.dev[2].fill_(600)
    call.score.fill_(MARK)
    g.replay()
    call.done()
    c2 = Cache(lens, 2, 4, 128, dtype, 64, seed=13, share=[(0, [1, 2], 890)])
    c2.lens = short
    c2.k, c2.v = [x[:, :, :n] for x, n in zip(c2.k, short)], [x[:, :, :n] for x, n in zip(c2.v, short)]
    call.c = c2
    out, tol, score, stol = reference(call)
    assert bool(((call.out.cpu().double() - out).abs() <= tol).all())
    for b, x in enumerate(short):
        assert bool(((call.score[b, :x].cpu().double() - score[b, :x]).abs() <= stol[b, :x]).all())
    c.t["len"].copy_(torch.tensor(lens, dtype=torch.int32))
    call.dev[2].fill_(890)
    call.score.fill_(MARK)
    g.replay()
    call.done()
    assert torch.equal(call.out, first[0]) and torch.equal(call.score, first[1])
