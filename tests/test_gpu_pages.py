"""Page pools: release, fork, writable and compact against a model of them in plain Python.

Everything here is whole numbers or bytes moved, so every comparison is exact."""
import random

import pytest
import torch

from paper_2609_03515_gb300 import DecodeCache, Q4Cache, ikv

pytestmark = pytest.mark.gpu


class Model:
    """The same books on the host: block table, counts, lengths, and each sequence's row numbers.  A
    row's content is a number, drawn when it is written; what the pages hold follows from it."""

    def __init__(self, c):
        self.c = c
        self.ps, self.cap, self.nb, self.P = c.page_size, c.cap, c.batch, c.num_pages
        self.table = [[0] * c.max_pages for _ in range(self.nb)]
        self.refs = [1] + [0] * (self.P - 1)
        self.len, self.next = [0] * self.nb, [0] * self.nb
        self.start = c.start.tolist()
        per = c.rows // self.nb
        self.pos = [[0] * self.cap for _ in range(self.nb * per)]
        self.rows = {}  # (page, offset, head) -> number

    def free(self):
        return [p for p in range(self.P) if self.refs[p] == 0]

    def release(self, extra=0):
        for b in range(self.nb):
            for p, e in enumerate(self.table[b]):
                inside = self.len[b] > 0 and (p + 1) * self.ps > self.start[b] and \
                    p * self.ps < self.start[b] + self.len[b] + extra
                if e and not inside:
                    self.refs[e] -= 1
                    self.table[b][p] = 0

    def fork(self, pairs):
        per = len(self.pos) // self.nb
        for s, d in pairs:
            self.table[d] = list(self.table[s])
            for e in self.table[d]:
                self.refs[e] += 1 if e else 0
            self.len[d], self.next[d], self.start[d] = self.len[s], self.next[s], self.start[s]
            for r in range(per):
                self.pos[d * per + r] = list(self.pos[s * per + r])

    def writable(self, ranges):
        """ranges: b -> (first, count); returns the pages lacking (nothing done then)."""
        asked = []
        for b in sorted(ranges):
            f, n = ranges[b]
            if n <= 0 or f < 0 or self.start[b] + f + n > self.cap:
                continue
            for p in range((self.start[b] + f) // self.ps, (self.start[b] + f + n - 1) // self.ps + 1):
                asked.append((b, p, self.table[b][p]))
        writers = {}
        for b, p, e in asked:
            if e and self.refs[e] > 1:
                writers.setdefault(e, []).append(b)
        need = [(b, p, e) for b, p, e in asked if not e or (
            self.refs[e] > 1 and not (len(writers[e]) == self.refs[e] and max(writers[e]) == b))]
        free = self.free()
        if len(need) > len(free):
            return len(need) - len(free)
        for (b, p, e), to in zip(need, free):
            self.table[b][p] = to
            self.refs[to] = 1
            if e:
                self.refs[e] -= 1
                for j in range(self.len[b]):
                    if (self.start[b] + j) // self.ps == p:
                        for g in range(self.c.kv_heads):
                            o = (self.start[b] + j) % self.ps
                            self.rows[to, o, g] = self.rows[e, o, g]
        return 0

    def compact(self, keep):
        """keep: b -> a list for every utility row, or None."""
        per = len(self.pos) // self.nb
        plan, total = {}, 0
        for b in range(self.nb):
            if keep.get(b) is None:
                continue
            n = len(keep[b][0])
            f = min(next((j for j in range(n) if k[j] != j), n) for k in keep[b])
            end = -(-(self.start[b] + n) // self.ps)
            begin = end if f == n else (self.start[b] + f) // self.ps
            plan[b] = (n, begin, end)
            total += end - begin
        free = self.free()
        if total > len(free):
            return total - len(free)
        for b, (n, begin, end) in plan.items():
            old = list(self.table[b])
            for p in range(begin, end):
                to = free.pop(0)
                for o in range(self.ps):
                    j = p * self.ps + o - self.start[b]
                    if 0 <= j < n:
                        for g in range(self.c.kv_heads):
                            k = self.start[b] + keep[b][g if per > 1 else 0][j]
                            self.rows[to, o, g] = self.rows[old[k // self.ps], k % self.ps, g]
                self.table[b][p] = to
            for p in range(end, len(old)):
                self.table[b][p] = 0
            for p in range(begin, end):
                self.refs[self.table[b][p]] = 1
            for p in range(begin, len(old)):
                if old[p]:
                    self.refs[old[p]] -= 1
            for r in range(per):
                row = self.pos[b * per + r]
                row[:n] = [row[k] for k in keep[b][r]]
            self.len[b] = n
        return 0

    # ---- the device's side
    def write(self, ranges, rng):
        """Fill slots with numbers, on both sides: every byte of a row follows from its number."""
        c, per = self.c, len(self.pos) // self.nb
        where, nums = [], []
        for b, (f, n) in ranges.items():
            for j in range(f, f + n):
                e, o = self.table[b][(self.start[b] + j) // self.ps], (self.start[b] + j) % self.ps
                assert e and self.refs[e] == 1
                for g in range(c.kv_heads):
                    x = rng.randrange(1, 1 << 20)
                    self.rows[e, o, g] = x
                    where.append((e, g, o))
                    nums.append(x)
        if where:
            at, x = torch.tensor(where, device="cuda").T, torch.tensor(nums, device="cuda")
            for t in c.planes():
                for layer in range(c.layers):
                    t[layer, at[0], at[1], at[2]] = pattern(x, layer, t)
        for b, (f, n) in ranges.items():
            self.len[b] = max(self.len[b], f + n)
            for r in range(per):
                for j in range(f, f + n):
                    self.pos[b * per + r][j] = self.next[b] + j - f
            self.next[b] += n
        self.upload()

    def upload(self):
        c = self.c
        c.len.copy_(torch.tensor(self.len, dtype=torch.int32))
        c.next_pos.copy_(torch.tensor(self.next, dtype=torch.int32))
        c.pos.copy_(torch.tensor(self.pos, dtype=torch.int32))
        c.ema.copy_(c.pos.float() * 0.5)
        if c.vnorm is not None:
            c.vnorm.copy_((c.pos.view(1, self.nb, -1, self.cap) * 2.0).expand_as(c.vnorm))

    def compare(self):
        c, per = self.c, len(self.pos) // self.nb
        assert c.block_table.tolist() == self.table
        assert c.refs.tolist() == self.refs
        assert c.len.tolist() == self.len and c.next_pos.tolist() == self.next and c.start.tolist() == self.start
        pos, ema = c.pos.tolist(), c.ema.tolist()
        where, nums = [], []
        for b in range(self.nb):
            for r in range(b * per, (b + 1) * per):
                assert pos[r][:self.len[b]] == self.pos[r][:self.len[b]]
                assert ema[r][:self.len[b]] == [0.5 * x for x in self.pos[r][:self.len[b]]]
            if c.vnorm is not None:
                for g in range(c.kv_heads):
                    want = [2.0 * x for x in self.pos[b * per + (g if per > 1 else 0)][:self.len[b]]]
                    for layer in range(c.layers):
                        assert c.vnorm[layer, b, g, :self.len[b]].tolist() == want
            for j in range(self.len[b]):
                e, o = self.table[b][(self.start[b] + j) // self.ps], (self.start[b] + j) % self.ps
                assert e
                for g in range(c.kv_heads):
                    where.append((e, g, o))
                    nums.append(self.rows[e, o, g])
        if where:
            at, x = torch.tensor(where, device="cuda").T, torch.tensor(nums, device="cuda")
            for t in c.planes():
                for layer in range(c.layers):
                    assert torch.equal(t[layer, at[0], at[1], at[2]], pattern(x, layer, t))


def pattern(x, layer, t):
    """What a row numbered x holds in a layer of plane t."""
    n = t.shape[-1]
    y = (x[:, None] * 2654435761 + layer * 97 + torch.arange(n, device="cuda") * 131) >> 7
    return (y % 251).to(t.dtype)


def make(kind, nb, ps, d, kvh, gran, starts, pool, cap=120, layers=2, norms=False):
    cls, dtype = {"q4": (Q4Cache, ikv.IKV_BF16), "bf16": (DecodeCache, ikv.IKV_BF16), "f32": (DecodeCache, ikv.IKV_F32)}[kind]
    c = cls(nb, layers, kvh, kvh, d, cap, dtype=dtype, page_size=ps, granularity=gran, pool_pages=pool,
            value_norms=norms)
    c.start.copy_(torch.tensor(starts, dtype=torch.int32))
    return c


CASES = [("bf16", 16, 128, 2, 0, False), ("f32", 7, 64, 1, 0, True), ("q4", 16, 128, 3, 1, False),
         ("q4", 32, 64, 2, 0, False), ("bf16", 1, 64, 2, 1, True), ("f32", 100, 128, 2, 1, False)]


@pytest.mark.parametrize("kind,ps,d,kvh,gran,norms", CASES)
@pytest.mark.parametrize("seed", [0, 1])
def test_random_life_of_a_pool(kind, ps, d, kvh, gran, norms, seed):
    """Sequences that begin, grow, fork, are compacted, cut and end, while pages run short now and then."""
    rng = random.Random(100 * seed + ps)
    nb = 6
    starts = [rng.choice([0, 0, 3, 2 * ps + 1]) if 2 * ps + 1 < 40 else 0 for _ in range(nb)]
    c = make(kind, nb, ps, d, kvh, gran, starts, pool=max(8, 330 // ps), norms=norms)
    m = Model(c)
    per = c.rows // nb
    ws = c.pages_workspace()
    lacking = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    short = cow = 0
    for step in range(60):
        what = rng.choice(["grow", "grow", "grow", "fork", "fork", "compact", "compact", "cut", "end", "release"])
        if what == "grow":
            ranges = {b: (m.len[b], rng.choice([1, 1, 2, ps, 2 * ps + 3])) for b in range(nb) if rng.random() < 0.7}
            ranges = {b: r for b, r in ranges.items() if m.start[b] + r[0] + r[1] <= m.cap}
            if not ranges:
                continue
            most = max(n for _, n in ranges.values())
            first = i32([ranges[b][0] if b in ranges else -1 for b in range(nb)])
            count = i32([ranges.get(b, (0, 0))[1] for b in range(nb)])
            held = [list(t) for t in m.table]
            lack = m.writable(ranges)
            ikv.ikv_pages_writable(shape, cache, pages, first, count, most, lacking, ws, ws.numel())
            assert int(lacking) == lack and ikv.ikv_device_status() == (64 if lack else 0)
            short += lack > 0
            cow += any(a and a != b for r0, r1 in zip(held, m.table) for a, b in zip(r0, r1))
            m.compare()
            if not lack:
                m.write(ranges, rng)
        elif what == "fork":
            empty = [b for b in range(nb) if not any(m.table[b])]
            full = [b for b in range(nb) if m.len[b] > 0]
            pairs = [(rng.choice(full), b) for b in empty if full and rng.random() < 0.7]
            m.fork(pairs)
            ikv.ikv_pages_fork(shape, cache, pages, len(pairs), i32([s for s, _ in pairs]), i32([d for _, d in pairs]),
                               c.ema)
        elif what in ("compact", "cut"):
            keep, kl, kp = {}, [], torch.zeros(c.rows, c.cap, dtype=torch.int32)
            for b in range(nb):
                n = rng.randint(0, m.len[b]) if rng.random() < 0.8 else None
                if n is None:
                    kl += [-1] * per
                    continue
                f = n if what == "cut" else rng.randint(0, n)
                keep[b] = [list(range(f)) + sorted(rng.sample(range(f, m.len[b]), n - f)) for _ in range(per)]
                for r in range(per):
                    kp[b * per + r, :n] = torch.tensor(keep[b][r], dtype=torch.int32)
                kl += [n] * per
            lack = m.compact(keep)
            ikv.ikv_pages_compact(shape, cache, pages, kp.cuda(), i32(kl), c.ema, lacking, ws, ws.numel())
            assert int(lacking) == lack and ikv.ikv_device_status() == (64 if lack else 0)
            short += lack > 0
        elif what == "end":
            b = rng.randrange(nb)
            m.len[b] = 0
            c.len[b] = 0
            m.release()
            ikv.ikv_pages_release(shape, cache, pages, 0)
        else:
            extra = rng.choice([0, 1, ps])
            m.release(extra)
            ikv.ikv_pages_release(shape, cache, pages, extra)
        m.compare()
        assert all(r >= 0 for r in m.refs) and sum(m.refs) == 1 + sum(e > 0 for t in m.table for e in t)
    assert cow or ps == 1
    assert ikv.ikv_device_status() == 0


@pytest.mark.parametrize("writers,kept", [((0, 1, 3), 2), ((0, 1, 2, 3), 3)])
def test_who_keeps_a_shared_page(writers, kept):
    """A page of four: three that write copy it; of four, the last goes on in it."""
    c = make("bf16", 4, 16, 64, 1, 0, [0] * 4, pool=4)
    m, rng = Model(c), random.Random(3)
    ws = c.pages_workspace()
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    m.writable({0: (0, 5)})
    ikv.ikv_pages_writable(shape, cache, pages, None, i32([5, 0, 0, 0]), 5, None, ws, ws.numel())
    m.compare()
    m.write({0: (0, 5)}, rng)
    m.fork([(0, 1), (0, 2), (0, 3)])
    ikv.ikv_pages_fork(shape, cache, pages, 3, i32([0, 0, 0]), i32([1, 2, 3]), c.ema)
    m.compare()
    m.writable({b: (5, 1) for b in writers})
    ikv.ikv_pages_writable(shape, cache, pages, i32([5 if b in writers else -1 for b in range(4)]), None, 1, None, ws,
                           ws.numel())
    m.compare()
    assert c.refs.tolist() == [1, 1, 1, 1, 1] and c.block_table[kept, 0] == 1
    # each has a page of its own now: nothing is left to do
    ikv.ikv_pages_writable(shape, cache, pages, None, None, 1, None, ws, ws.numel())
    m.compare()
    assert ikv.ikv_device_status() == 0


def test_slots_past_the_space_and_bad_forks():
    c = make("bf16", 2, 16, 64, 1, 0, [0, 8], pool=20, cap=64)
    ws = c.pages_workspace()
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c.len.copy_(i32([60, 50]))
    ikv.ikv_pages_writable(shape, cache, pages, None, None, 5, None, ws, ws.numel())  # 60 + 5 > 64
    assert ikv.ikv_device_status() == 4
    assert c.block_table.tolist() == [[0, 0, 0, 0], [0, 0, 0, 1]]
    table, refs = c.block_table.clone(), c.refs.clone()
    ikv.ikv_pages_fork(shape, cache, pages, 2, i32([7, 1]), i32([0, -1]), None)
    assert ikv.ikv_device_status() == 128
    assert torch.equal(table, c.block_table) and torch.equal(refs, c.refs)


@pytest.mark.parametrize("pool", [3000, 40000])
def test_free_pages_of_a_large_pool(pool):
    """The lowest free pages of a pool longer than one pass of the search, most of it taken."""
    c = DecodeCache(3, 1, 1, 1, 64, 16 * 700, dtype=ikv.IKV_BF16, page_size=16, pool_pages=pool)
    gen = torch.Generator(device="cuda").manual_seed(pool)
    taken = torch.rand(pool + 1, generator=gen, device="cuda") < 0.7
    taken[0] = True
    c.refs.copy_(taken.to(torch.int32))
    free = (~taken).nonzero()[:, 0].tolist()
    ws = c.pages_workspace()
    count = torch.tensor([16 * 300, 1, 16 * 250 - 3], dtype=torch.int32, device="cuda")
    ikv.ikv_pages_writable(c.shape(), c.cache(0), c.pages(), None, count, 16 * 300, None, ws, ws.numel())
    assert ikv.ikv_device_status() == 0
    assert c.block_table[0, :300].tolist() == free[:300] and int(c.block_table[1, 0]) == free[300]
    assert c.block_table[2, :250].tolist() == free[301:551] and int(c.refs.sum()) == pool + 1 - len(free) + 551


@pytest.mark.parametrize("nb,idle", [(250, 0), (300, 0), (300, 3), (1100, 0)])
def test_many_sequences_share_and_leave_a_page(nb, idle):
    """More requests than one CTA plans in shared memory, and more sequences than it has threads: all
    write a shared page (the last keeps it, or nobody while some are idle), then all are compacted."""
    c = make("bf16", nb, 16, 64, 1, 0, [0] * nb, pool=3 * nb, cap=48, layers=1)
    m, rng = Model(c), random.Random(nb)
    ws = c.pages_workspace()
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    m.writable({0: (0, 20)})
    ikv.ikv_pages_writable(shape, cache, pages, None, i32([20] + [0] * (nb - 1)), 20, None, ws, ws.numel())
    m.compare()
    m.write({0: (0, 20)}, rng)
    m.fork([(0, b) for b in range(1, nb)])
    ikv.ikv_pages_fork(shape, cache, pages, nb - 1, i32([0] * (nb - 1)), i32(list(range(1, nb))), c.ema)
    m.compare()
    who = {b: (20, 2) for b in range(nb - idle)}
    m.writable(who)
    ikv.ikv_pages_writable(shape, cache, pages, None, i32([2 if b in who else 0 for b in range(nb)]), 2, None, ws, ws.numel())
    m.compare()
    kept = c.block_table[:, 1].tolist().count(2)
    assert kept == (1 if idle == 0 else idle) and c.block_table[0, 0] == 1 and int(c.refs[1]) == nb
    m.write(who, rng)
    keep, kp, kl = {}, torch.zeros(nb, c.cap, dtype=torch.int32), []
    for b in range(nb):
        n = rng.choice([17, 5, m.len[b]])
        keep[b] = [sorted(rng.sample(range(m.len[b]), n))]
        kp[b, :n] = torch.tensor(keep[b][0], dtype=torch.int32)
        kl.append(n)
    assert m.compact(keep) == 0
    ikv.ikv_pages_compact(shape, cache, pages, kp.cuda(), i32(kl), c.ema, None, ws, ws.numel())
    m.compare()
    assert ikv.ikv_device_status() == 0


def test_nothing_to_do():
    """No slots asked for, no forks, empty sequences: nothing changes, and lacking says 0."""
    c = make("q4", 3, 16, 64, 1, 0, [0] * 3, pool=5)
    ws = c.pages_workspace()
    shape, cache, pages = c.shape(), c.cache(0), c.pages()
    lacking = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    ikv.ikv_pages_writable(shape, cache, pages, None, None, 0, lacking, ws, ws.numel())
    assert int(lacking) == 0
    lacking.fill_(9)
    ikv.ikv_pages_fork(shape, cache, pages, 0, None, None, None)
    ikv.ikv_pages_release(shape, cache, pages, 3)
    keep, kl = torch.zeros(3, c.cap, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    ikv.ikv_pages_compact(shape, cache, pages, keep, kl, None, lacking, ws, ws.numel())
    assert int(lacking) == 0 and ikv.ikv_device_status() == 0
    assert not c.block_table.any() and c.refs.tolist() == [1, 0, 0, 0, 0, 0] and not c.len.any()


@pytest.mark.parametrize("kind,ps,nb", [("bf16", 16, 5), ("q4", 48, 300)])
def test_workspace_and_other_pages_stay_as_they_are(kind, ps, nb):
    """A pattern behind the workspace, and the contents of every page that a call does not hand out."""
    c = make(kind, nb, ps, 64, 2, 0, [0] * nb, pool=4 * nb, cap=2 * ps, layers=2)
    m, rng = Model(c), random.Random(nb)
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    n = ikv.ikv_pages_workspace_size(shape, cache, pages)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")

    def untouched(call):
        before, free = [t.clone() for t in c.planes()], c.refs == 0
        call()
        same = ~(free & (c.refs > 0))
        for t, was in zip(c.planes(), before):
            assert torch.equal(t[:, same], was[:, same])
        assert bool((ws[n:] == 0x5A).all()) and ikv.ikv_device_status() == 0

    want = {b: (0, ps + 1) for b in range(0, nb, 2)}
    m.writable(want)
    untouched(lambda: ikv.ikv_pages_writable(shape, cache, pages, None, i32([ps + 1 if b in want else 0 for b in range(nb)]),
                                             ps + 1, None, ws, n))
    m.write(want, rng)
    pairs = [(b - 1, b) for b in range(1, nb, 2)]
    m.fork(pairs)
    untouched(lambda: ikv.ikv_pages_fork(shape, cache, pages, len(pairs), i32([s for s, _ in pairs]), i32([d for _, d in pairs]),
                                         c.ema))
    m.writable({b: (ps + 1, 1) for b in range(nb)})
    untouched(lambda: ikv.ikv_pages_writable(shape, cache, pages, None, None, 1, None, ws, n))
    m.compare()
    keep = {b: [[0, 1] + list(range(3, ps + 1))] for b in range(0, nb, 3)}
    kp = torch.zeros(c.rows, c.cap, dtype=torch.int32)
    for b, k in keep.items():
        kp[b, :len(k[0])] = torch.tensor(k[0], dtype=torch.int32)
    assert m.compact(keep) == 0
    kp, kl = kp.cuda(), i32([len(keep[b][0]) if b in keep else -1 for b in range(nb)])
    untouched(lambda: ikv.ikv_pages_compact(shape, cache, pages, kp, kl, c.ema, None, ws, n))
    m.compare()


def test_compaction_of_many_table_entries():
    """Block tables too long for the plan to write: sequences compacted, cut, emptied and left alone."""
    nb, ps = 90, 7
    c = make("f32", nb, ps, 64, 1, 0, [b % 9 for b in range(nb)], pool=900, cap=700, layers=1)
    assert nb * c.max_pages > 8192
    m, rng = Model(c), random.Random(8)
    ws = c.pages_workspace()
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = {b: (0, 10 + (11 * b) % 25) for b in range(nb)}
    m.writable(lens)
    ikv.ikv_pages_writable(shape, cache, pages, None, i32([n for _, n in lens.values()]), 40, None, ws, ws.numel())
    m.compare()
    m.write(lens, rng)
    keep, kp, kl = {}, torch.zeros(nb, c.cap, dtype=torch.int32), []
    for b in range(nb):
        n = [m.len[b], 0, 5, m.len[b] - 3, None][b % 5]
        kl.append(-1 if n is None else n)
        if n is not None:
            keep[b] = [list(range(n)) if b % 10 < 5 else sorted(rng.sample(range(m.len[b]), n))]
            kp[b, :n] = torch.tensor(keep[b][0], dtype=torch.int32)
    assert m.compact(keep) == 0
    ikv.ikv_pages_compact(shape, cache, pages, kp.cuda(), i32(kl), c.ema, None, ws, ws.numel())
    m.compare()
    assert ikv.ikv_device_status() == 0


def test_compaction_past_the_slot_space():
    """A keep_len that does not fit behind its start is cut to what does, and says so."""
    c = make("bf16", 2, 16, 64, 1, 0, [8, 0], pool=20, cap=64)
    ws = c.pages_workspace()
    shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ikv.ikv_pages_writable(shape, cache, pages, None, i32([56, 30]), 56, None, ws, ws.numel())
    c.len.copy_(i32([56, 30]))
    table, refs = c.block_table.clone(), c.refs.clone()
    keep = torch.arange(64, dtype=torch.int32, device="cuda").repeat(2, 1)
    ikv.ikv_pages_compact(shape, cache, pages, keep, i32([64, 30]), c.ema, None, ws, ws.numel())
    assert ikv.ikv_device_status() == 4
    assert c.len.tolist() == [56, 30]
    assert torch.equal(table, c.block_table) and torch.equal(refs, c.refs)


@pytest.mark.parametrize("kind,ps,d,kvh,norms", [("bf16", 64, 128, 3, False), ("f32", 64, 128, 5, True), ("f32", 33, 128, 7, False),
                                                 ("q4", 128, 128, 8, False)])
def test_compactions_cut_into_some_of_the_heads(kind, ps, d, kvh, norms):
    """Rows long enough that few pages are moved in items of fewer heads than share their moves."""
    test_random_life_of_a_pool(kind, ps, d, kvh, 0, norms, 2)


def test_copies_of_a_row_and_of_many():
    """Writable pages whose copies are all short (a warp's each), and one long among them."""
    for longest in (1, 16, 17, 64):
        c = make("bf16", 4, 64, 64, 2, 0, [0, 0, 0, 0], pool=12, cap=128)
        m, rng = Model(c), random.Random(longest)
        ws = c.pages_workspace()
        shape, cache, pages = c.shape(), c.cache(c.cap), c.pages()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        first = {0: (0, 1), 1: (0, longest)}
        m.writable(first)
        ikv.ikv_pages_writable(shape, cache, pages, i32([0, 0, -1, -1]), i32([1, longest, 0, 0]), 64, None, ws, ws.numel())
        m.write(first, rng)
        m.fork([(0, 2), (1, 3)])
        ikv.ikv_pages_fork(shape, cache, pages, 2, i32([0, 1]), i32([2, 3]), c.ema)
        n = min(longest, 63)  # the page's last slot at the latest
        m.writable({2: (1, 1), 3: (n, 1)})
        ikv.ikv_pages_writable(shape, cache, pages, i32([-1, -1, 1, n]), None, 1, None, ws, ws.numel())
        m.compare()
        assert ikv.ikv_device_status() == 0
