"""ikv_window_attend against a 64-bit evaluation: lengths from one token on, odd sizes, windows and sinks
that cut tiles anywhere, dead slots, rows that see nothing, NaN wherever no query looks."""
import math

import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import DT, MARK, Cache, attention, window_seen

pytestmark = pytest.mark.gpu


def run(c, counts, window, sinks, layer=1, row0=None, max_count=None, q_pad=0, out_pad=0, seed=5, stream=None, q=None):
    """out (on the host), the queries, and each sequence's first row"""
    nb, w = len(c.lens), c.h * c.d
    max_count = max(counts) if max_count is None else max_count
    if row0 is None:
        row0 = [sum(counts[:b]) for b in range(nb)]
    rows = max([r + n for r, n in zip(row0, counts)] + [1]) + 1
    if q is None:
        q = torch.randn(rows, w + q_pad, generator=torch.Generator().manual_seed(seed)).to(DT[c.dtype])
    out = torch.full((rows, w + out_pad), MARK, dtype=DT[c.dtype], device="cuda")
    qd, r0, cn = q.cuda(), torch.tensor(row0, dtype=torch.int32).cuda(), torch.tensor(counts, dtype=torch.int32).cuda()
    win = ikv.ikv_window(window, sinks, r0.data_ptr(), cn.data_ptr(), max_count, (w + q_pad) if q_pad else 0,
                         (w + out_pad) if out_pad else 0)
    n = ikv.ikv_window_workspace_size(c.shape(), c.cache(), win)
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    ikv.ikv_window_attend(c.shape(), c.cache(), win, layer, qd, out, ws, n, stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 0
    assert bool((ws[n:] == 0xA5).all())
    return out.cpu(), q, row0


def check(c, counts, window, sinks, layer=1, max_count=None, **kw):
    out, q, row0 = run(c, counts, window, sinks, layer, max_count=max_count, **kw)
    untouched = torch.ones_like(out, dtype=torch.bool)
    for b, n in enumerate(c.lens):
        cnt = min(counts[b], max_count) if max_count is not None else counts[b]
        if cnt == 0:
            continue
        untouched[row0[b]:row0[b] + cnt, :c.h * c.d] = False
        seen_all = window_seen(n, cnt, 0, cnt, window, sinks)
        for i in range(c.g):
            seen = seen_all & c.alive(b, i)[None] if c.dead else seen_all
            for x in range(c.G):
                h = i * c.G + x
                cols = slice(h * c.d, (h + 1) * c.d)
                ref, _, tol, _ = attention(c, layer, b, i, q[row0[b]:row0[b] + cnt, cols], seen)
                got = out[row0[b]:row0[b] + cnt, cols].double()
                worst = ((got - ref).abs() / tol).nan_to_num(nan=math.inf).amax().item()
                assert worst <= 1.0, (b, h, worst)
    assert bool((out[untouched] == MARK).all())


def counts_of(lens, kind):
    return {"one": [1] * len(lens), "all": list(lens), "some": [max(1, n // 3) for n in lens],
            "few": [min(n, 5) for n in lens]}[kind]


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("bf16", 20), ("f32", 16)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 7, 8])
@pytest.mark.parametrize("kind", ["one", "few", "all"])
@pytest.mark.parametrize("hidden", [math.nan, 9.0])
def test_shapes(dtype, page, d, group, kind, hidden):
    lens = [300, 1, 129, 57]
    c = Cache(lens, 2, group, d, dtype, page, seed=1).device(hidden)
    check(c, counts_of(lens, kind), 100, 3)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 20), ("f32", 16)])
@pytest.mark.parametrize("window", [0, 1, 2, 63, 64, 128, 129, 200, 5000, 2**31 - 1])
@pytest.mark.parametrize("sinks", [0, 1, 4, 130, 2**31 - 1])
@pytest.mark.parametrize("hidden", [math.nan, 9.0])
def test_windows(dtype, page, window, sinks, hidden):
    lens = [401, 128, 6]
    c = Cache(lens, 1, 4, 128, dtype, page, seed=2, starts=[0, 5, 77]).device(hidden)
    for kind in ("one", "some", "all"):
        check(c, counts_of(lens, kind), window, sinks)


@pytest.mark.parametrize("dtype,page", [("bf16", 8), ("bf16", 24), ("bf16", 128), ("bf16", 256), ("bf16", 1), ("f32", 5)])
@pytest.mark.parametrize("start", [0, 1, 127, 130])
@pytest.mark.parametrize("hidden", [math.nan, 9.0])
def test_pages_and_starts(dtype, page, start, hidden):
    lens = [260, 33, 512]
    c = Cache(lens, 2, 2, 128, dtype, page, seed=3, starts=[start, 0, start + 3]).device(hidden)
    check(c, [7, 33, 140], 90, 5)
    check(c, [1, 1, 1], 90, 5, layer=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gran", ["seq", "kvhead"])
@pytest.mark.parametrize("dead", [0.3, 0.97, 1.0])
@pytest.mark.parametrize("hidden", [math.nan, 9.0])
def test_dead_slots_are_not_seen(dtype, gran, dead, hidden):
    lens = [300, 40, 131]
    c = Cache(lens, 2, 4, 128, dtype, 16, seed=4, dead=dead, gran=gran, starts=[3, 0, 64])
    if gran == "seq" and math.isnan(hidden):  # dead rows hold NaN
        for b in range(len(lens)):
            c.k[b][:, :, ~c.alive(b, 0)] = math.nan
            c.v[b][:, :, ~c.alive(b, 0)] = math.inf
    c.device(hidden)
    check(c, [300, 40, 131], 50, 4)
    check(c, [1, 1, 1], 50, 4)
    check(c, [9, 9, 9], 0, 0)


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("bf16", 20), ("f32", 64)])
def test_what_a_query_does_not_see_never_reaches_it(dtype, page):
    """A token in the middle is NaN in K and infinite in V: queries that see it are NaN, the others are right."""
    n, bad, window, sinks = 300, 150, 60, 4
    c = Cache([n], 1, 2, 128, dtype, page, seed=6)
    clean = Cache([n], 1, 2, 128, dtype, page, seed=6)
    c.k[0][:, :, bad] = math.nan
    c.v[0][:, :, bad] = math.inf
    c.device()
    for count in (n, 1, 100):
        out, q, _ = run(c, [count], window, sinks)
        for i in range(count):
            p = n - count + i
            got = out[i].double()
            if p >= bad > p - window:
                assert bool(got.isnan().all()), p
            else:
                seen = window_seen(n, count, i, i + 1, window, sinks)
                for h in range(2):
                    cols = slice(h * 128, (h + 1) * 128)
                    ref, _, tol, _ = attention(clean, 1, 0, 0, q[i:i + 1, cols], seen)
                    assert bool(((got[cols] - ref[0]).abs() <= tol[0]).all()), p


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_value_that_is_seen_stays_infinite(dtype):
    c = Cache([200], 1, 1, 128, dtype, 64, seed=7)
    c.v[0][1, 0, 100, 5] = math.inf
    c.device()
    out, _, _ = run(c, [200], 0, 0)
    assert bool((out[100:200, 5] == math.inf).all())
    assert bool(out[:200].float()[:, [0, 1, 4, 6, 127]].isfinite().all()) and bool(out[:100, :128].float().isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_sequences_and_counts(dtype):
    """No tokens, no queries, more queries than tokens (those in front of the first slot see nothing), counts
    beyond max_count."""
    lens = [0, 50, 3, 20]
    c = Cache(lens, 2, 4, 64, dtype, 16, seed=8).device()
    out, q, row0 = run(c, [2, 0, 9, 4], 10, 1)
    assert bool((out[0:2] == 0).all()) and bool((out[2:8] == 0).all())  # (both of an empty sequence; six of nine)
    check(c, [0, 50, 3, 20], 10, 1)
    check(c, [0, 9, 3, 20], 10, 1, max_count=9)


def test_rows_apart_and_strided():
    """Queries that are slices of a projection's rows, output rows with gaps, in another order than the sequences."""
    lens = [140, 31, 60]
    for dtype in ("bf16", "f32"):
        c = Cache(lens, 2, 4, 64, dtype, 16, seed=9).device()
        check(c, [70, 31, 1], 40, 2, row0=[35, 0, 120], q_pad=16, out_pad=8)


def test_null_rows_and_counts():
    lens = [30, 30]
    c = Cache(lens, 1, 1, 64, "bf16", 16, seed=10).device()
    q = torch.randn(10, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    win = ikv.ikv_window(8, 0, None, None, 5, 0, 0)
    n = ikv.ikv_window_workspace_size(c.shape(), c.cache(), win)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    ikv.ikv_window_attend(c.shape(), c.cache(), win, 0, q, out, ws, n)
    torch.cuda.synchronize()
    ref, _, _ = run(c, [5, 5], 8, 0, layer=0, q=torch.cat([q.cpu(), q.cpu()[:1]]))
    assert torch.equal(out.cpu(), ref[:10])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_contexts_split_over_the_gpu(dtype):
    """One token and a chunk of 300 over 20000 slots: every share's border inside a pair."""
    c = Cache([20000], 2, 4, 128, dtype, 64, seed=11, layers=1).device(9.0)
    for counts, window in (([1], 0), ([1], 9999), ([300], 0)):
        check(c, counts, window, 4, layer=0)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 48), ("f32", 16)])
def test_a_slot_space_that_is_full(dtype, page):
    """The last slot is the slot space's last: nothing behind the block table is looked up."""
    lens = [6 * page - 3, 6 * page - 17, 1]
    c = Cache(lens, 2, 4, 128, dtype, page, seed=15, starts=[3, 17, 6 * page - 1], extra_pages=0).device()
    assert c.cap == 6 * page
    for kind in ("one", "some", "all"):
        check(c, counts_of(lens, kind), 40, 5)
        check(c, counts_of(lens, kind), 0, 0)


def test_many_short_sequences():
    lens = [1 + (i * 37) % 90 for i in range(300)]
    c = Cache(lens, 1, 8, 64, "bf16", 16, seed=12, layers=1).device()
    check(c, [1 + i % min(7, n) for i, n in enumerate(lens)], 33, 2, layer=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(dtype):
    """Logits of some hundred: the running maximum moves far, weights underflow."""
    c = Cache([700], 1, 4, 128, dtype, 64, seed=13, spread=40.0).device(9.0)
    check(c, [700], 0, 0)
    check(c, [2], 300, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replayed_from_a_graph_on_another_stream_and_twice_the_same(dtype):
    c = Cache([1000, 77], 2, 4, 128, dtype, 64, seed=14).device()
    first, q, _ = run(c, [40, 77], 200, 4)
    win_q, r0 = q.cuda(), torch.tensor([0, 40], dtype=torch.int32).cuda()
    cn = torch.tensor([40, 77], dtype=torch.int32).cuda()
    win = ikv.ikv_window(200, 4, r0.data_ptr(), cn.data_ptr(), 77, 0, 0)
    shape, cache = c.shape(), c.cache()
    n = ikv.ikv_window_workspace_size(shape, cache, win)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = torch.full_like(win_q, MARK)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        ikv.ikv_window_attend(shape, cache, win, 1, win_q, out, ws, n, st)
        st.synchronize()
        with torch.cuda.graph(g, stream=st):
            ikv.ikv_window_attend(shape, cache, win, 1, win_q, out, ws, n, torch.cuda.current_stream())
    for _ in range(3):
        out.fill_(MARK)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), first)
