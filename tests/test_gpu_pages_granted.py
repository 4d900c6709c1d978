"""What ikv_pages_writable grants: stores and appends that are enqueued behind a shortage touch no page
that is not their sequence's own."""
import random

import pytest
import torch
from test_gpu_q4 import quantise, values

from paper_2609_03515_gb300 import DecodeCache, Q4Cache, ikv

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(kind, nb, pool, cap=96, ps=16, starts=None):
    c = (Q4Cache if kind == "q4" else DecodeCache)(nb, 2, 4, 2, 64, cap, page_size=ps, pool_pages=pool)
    if starts:
        c.start.copy_(i32(starts))
    return c


def append(kind, c, x, slot=None):
    if kind == "q4":
        ikv.ikv_q4_append_token(c.shape(), c.cache(c.cap - 1), c.q4(), x, x, c.ema, 0, slot)
    else:
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        ikv.ikv_append_token(c.shape(), c.cache(c.cap - 1, granted=True), x, x, c.ema, 0, ws, ws.numel())


@pytest.mark.parametrize("kind", ["q4", "bf16"])
def test_a_shortage_leaves_the_rest_alone(kind):
    """Four samples of a prompt and two sequences of their own, in a pool with two free pages where
    four are wanted: nothing is copied; the one whose next slot lies in a page of its own goes on."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    c = make(kind, 6, 5)
    shape, cache, pages, ws = c.shape(), c.cache(c.cap - 1, granted=True), c.pages(), c.pages_workspace()
    lacking, slot = i32([9]), i32([7] * 6)
    ikv.ikv_pages_writable(shape, cache, pages, i32([0, -1, -1, -1, 0, 0]), i32([5, 0, 0, 0, 7, 16]), 16, lacking, ws, ws.numel())
    assert int(lacking) == 0 and c.writable.tolist() == [[0, 5], [0, 0], [0, 0], [0, 0], [0, 7], [0, 16]]
    for t in c.planes():
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda").mul(20).to(t.dtype) if t.is_floating_point()
                else torch.randint(0, 256, t.shape, generator=gen, device="cuda").to(t.dtype))
    c.len.copy_(i32([5, 0, 0, 0, 7, 16]))
    c.next_pos.copy_(c.len)
    ikv.ikv_pages_fork(shape, cache, pages, 3, i32([0, 0, 0]), i32([1, 2, 3]), c.ema)
    assert c.writable.tolist() == [[0, 0]] * 4 + [[0, 7], [0, 16]]
    # three copies and a page behind the last sequence's first: two are free
    ikv.ikv_pages_writable(shape, cache, pages, None, None, 1, lacking, ws, ws.numel())
    assert int(lacking) == 2 and ikv.ikv_device_status() == 64
    assert c.writable.tolist() == [[0, 0]] * 4 + [[0, 8], [0, 16]]
    held, books = [t.clone() for t in c.planes()], [t.clone() for t in (c.pos, c.ema, c.next_pos, c.block_table, c.refs)]
    x = torch.randn(2, 6, 2, 64, generator=gen, device="cuda").to(torch.bfloat16)
    append(kind, c, x, slot)
    if kind == "q4":
        assert slot.tolist() == [-1, -1, -1, -1, 7, -1]
        # a store that goes by its own list of slots
        rows = c.dense_rows(x.unsqueeze(2))
        ikv.ikv_q4_store(shape, cache, c.q4(), 0, 2, x, x, rows, i32([5, 5, 5, 5, 8, 16]), None, 1)
    assert ikv.ikv_device_status() == 256
    assert c.len.tolist() == [5, 5, 5, 5, 8, 16]
    own = int(c.block_table[4, 0])
    for t, was in zip(c.planes(), held):
        same = torch.ones(t.shape, dtype=torch.bool, device="cuda")
        same[:, own, :, 7] = False
        assert torch.equal(t[same], was[same]) and not torch.equal(t, was)
    for t, was in zip((c.pos, c.ema, c.next_pos, c.block_table, c.refs), books):
        rest = [0, 1, 2, 3, 5]
        assert torch.equal(t, was) if t.shape[0] != 6 else torch.equal(t[rest], was[rest])
    # pages come back: the same calls go through
    ikv.ikv_pages_writable(shape, cache, pages, i32([-1, 5, 5, -1, -1, -1]), None, 1, lacking, ws, ws.numel())
    assert int(lacking) == 0 and c.writable.tolist() == [[0, 0], [5, 6], [5, 6], [0, 0], [0, 8], [0, 16]]
    append(kind, c, x, slot)
    assert ikv.ikv_device_status() == 256 and c.len.tolist() == [5, 6, 6, 5, 8, 16]


@pytest.mark.parametrize("ps,nb,most,pool,scarce", [(16, 6, 20, 12, True), (32, 5, 3, 6, False), (48, 300, 60, 200, True)])
def test_grants_follow_the_pages(ps, nb, most, pool, scarce):
    """Random lives: a sequence's grant is what it was last given, with what touched it before, and all of its
    pages are the sequence's own; forks, compactions and releases take it back."""
    rng = random.Random(ps)
    starts = [rng.choice([0, 0, 2 * ps + 1]) for _ in range(nb)]
    c = make("q4", nb, pool, cap=5 * ps, ps=ps, starts=starts)
    shape, cache, pages, ws = c.shape(), c.cache(c.cap), c.pages(), c.pages_workspace()
    want = [[0, 0] for _ in range(nb)]
    short = 0
    for _ in range(50):
        what = rng.choice(["ask", "ask", "ask", "fork", "compact", "release"])
        lens, table = c.len.tolist(), c.block_table.tolist()
        if what == "ask":
            first = [rng.choice([-1, n, n, max(0, n - 2)]) for n in lens]
            count = [rng.choice([-1, 0, 1, 1, most, c.cap]) for _ in range(nb)]
            ikv.ikv_pages_writable(shape, cache, pages, i32(first), i32(count), most, None, ws, ws.numel())
            status = ikv.ikv_device_status()
            assert status & ~68 == 0
            short += status & 64 > 0
            table, refs = c.block_table.tolist(), c.refs.tolist()
            for b in range(nb):
                n = min(count[b], most)
                if first[b] < 0 or n <= 0:
                    continue
                s = starts[b] + first[b]
                own = s + n <= c.cap and all(table[b][p] and refs[table[b][p]] == 1
                                             for p in range(s // c.page_size, (s + n - 1) // c.page_size + 1))
                if own:
                    lo, hi = first[b], first[b] + n
                    if want[b][0] < want[b][1] and want[b][0] <= hi and lo <= want[b][1]:
                        lo, hi = min(lo, want[b][0]), max(hi, want[b][1])
                    want[b] = [lo, hi]
                    lens[b] = max(lens[b], first[b] + n)
            c.len.copy_(i32(lens))
        elif what == "fork":
            empty = [b for b in range(nb) if not any(table[b])]
            full = [b for b in range(nb) if lens[b] > 0]
            pairs = [(rng.choice(full), b) for b in empty if full and rng.random() < 0.5]
            ikv.ikv_pages_fork(shape, cache, pages, len(pairs), i32([s for s, _ in pairs]), i32([d for _, d in pairs]), None)
            for s, d in pairs:
                want[s], want[d] = [0, 0], [0, 0]
                starts[d] = starts[s]
        elif what == "compact":
            keep = torch.arange(c.cap, dtype=torch.int32, device="cuda").repeat(nb, 1)
            n = [rng.choice([-1, rng.randint(0, x)]) for x in lens]
            ikv.ikv_pages_compact(shape, cache, pages, keep, i32(n), None, None, ws, ws.numel())
            assert ikv.ikv_device_status() == 0
            want = [w if x < 0 else [0, 0] for w, x in zip(want, n)]
        else:
            for b in range(nb):
                if rng.random() < 0.2:
                    c.len[b] = 0
            ikv.ikv_pages_release(shape, cache, pages, rng.choice([0, 1]))
            after = c.block_table.tolist()
            want = [w if x == y else [0, 0] for w, x, y in zip(want, table, after)]
        assert c.writable.tolist() == want
        table, refs = c.block_table.tolist(), c.refs.tolist()
        for b, (lo, hi) in enumerate(want):
            for p in range((starts[b] + lo) // ps, (starts[b] + hi - 1) // ps + 1) if lo < hi else ():
                assert table[b][p] > 0 and refs[table[b][p]] == 1
    assert short or not scarce


def test_one_token_each_in_a_graph():
    """The decode loop's calls, captured: a sequence that finds no page stands still until one is free."""
    c = make("q4", 3, 4)
    shape, cache, pages, ws = c.shape(), c.cache(c.cap - 1), c.pages(), c.pages_workspace()
    x, slot = torch.randn(2, 3, 2, 64, device="cuda").to(torch.bfloat16), i32([0, 0, 0])

    def step():
        ikv.ikv_pages_writable(shape, cache, pages, None, None, 1, None, ws, ws.numel(), torch.cuda.current_stream())
        ikv.ikv_q4_append_token(shape, cache, c.q4(), x, x, c.ema, 0, slot, torch.cuda.current_stream())

    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step()
    st.synchronize()
    for _ in range(15):
        g.replay()
    assert c.len.tolist() == [16, 16, 16] and ikv.ikv_device_status() == 0
    g.replay()  # three pages are wanted, one is free: none is handed out
    torch.cuda.synchronize()
    assert c.len.tolist() == [16, 16, 16] and ikv.ikv_device_status() == 64 + 256 and int((c.refs[1:] > 0).sum()) == 3
    c.len[1] = 0
    ikv.ikv_pages_release(shape, cache, pages, 0)
    g.replay()  # now two are, for the two that go on; the third starts anew and takes none
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 64 + 256 and c.len.tolist() == [16, 0, 16]
    c.len[2] = 0
    ikv.ikv_pages_release(shape, cache, pages, 0)
    g.replay()
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 0 and c.len.tolist() == [17, 1, 1]


def test_chunks_are_granted_together():
    """A prompt in two pieces, both granted before either is stored; a piece that touches neither is refused."""
    c = make("q4", 1, 6)
    shape, cache, pages, ws = c.shape(), c.cache(c.cap - 1), c.pages(), c.pages_workspace()
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(2, 1, 40, 2, 64, generator=gen, device="cuda").to(torch.bfloat16)
    for first, n in ((0, 20), (20, 20)):
        ikv.ikv_pages_writable(shape, cache, pages, i32([first]), None, n, None, ws, ws.numel())
    assert c.writable.tolist() == [[0, 40]]
    for first, n in ((0, 20), (20, 20)):
        part = x[:, :, first:first + n]
        ikv.ikv_q4_store(shape, cache, c.q4(), 0, 2, part, part, c.dense_rows(part), i32([first]), None, n)
    assert ikv.ikv_device_status() == 0
    back, other = torch.zeros_like(x), torch.zeros_like(x)
    ikv.ikv_q4_load(shape, cache, c.q4(), 0, 2, back, other, c.dense_rows(back), i32([0]), None, 40)
    want = values(*quantise(x)).to(torch.bfloat16)
    assert torch.equal(back, want) and torch.equal(other, want)
    held = [t.clone() for t in c.planes()]
    ikv.ikv_q4_store(shape, cache, c.q4(), 0, 2, x, x, c.dense_rows(x), i32([30]), None, 20)  # 30 .. 49
    assert ikv.ikv_device_status() == 256 and all(torch.equal(t, was) for t, was in zip(c.planes(), held))
