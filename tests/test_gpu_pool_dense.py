"""16- and 32-bit caches on pages from a pool, under the framework's own decode calls: the same outputs and
the same cache, bit for bit, as on pages that each sequence owns for good."""
import random

import pytest
import torch

from paper_2609_03515_gb300 import DecodeCache, ikv

pytestmark = pytest.mark.gpu

DT = {ikv.IKV_F32: torch.float32, ikv.IKV_BF16: torch.bfloat16}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(pool, nb, kvh, G, d, dtype, ps, gran, cap=160, layers=2):
    return DecodeCache(nb, layers, G * kvh, kvh, d, cap, dtype=dtype, page_size=ps, granularity=gran, pool_pages=pool,
                       value_norms=True)


class Pair:
    """The same sequences twice: in a pool, with the page calls in front of whatever writes, and without."""

    def __init__(self, *shape):
        self.p, self.d = make(60 * 64 // shape[5], *shape), make(None, *shape)
        self.shape, self.pages, self.ws = self.p.shape(), self.p.pages(), self.p.pages_workspace()
        self.gen = torch.Generator(device="cuda").manual_seed(shape[5])
        self.lacking = i32([0])

    def both(self):
        return self.p, self.d

    def writable(self, first, count):
        ikv.ikv_pages_writable(self.shape, self.p.cache(0, granted=True), self.pages, first, count, self.p.cap, self.lacking, self.ws,
                               self.ws.numel())
        assert int(self.lacking) == 0

    def prompt(self, lens):
        self.writable(torch.zeros_like(self.p.len), i32(lens))
        for b, n in enumerate(lens):
            for layer in range(self.p.layers):
                for g in range(self.p.kv_heads):
                    for kv in ("k", "v"):
                        x = torch.randn(n, self.p.head_dim, generator=self.gen, device="cuda")
                        for c in self.both():
                            c.scatter(getattr(c, kv), b, layer, g, x)
        for c in self.both():
            c.len.copy_(i32(lens))
            c.next_pos.copy_(c.len)
            c.pos.copy_(torch.arange(c.cap, dtype=torch.int32, device="cuda").expand_as(c.pos))
            ikv.ikv_value_norms(c.shape(), c.cache(c.cap))

    def fork(self, src, dst):
        p, d = self.both()
        ikv.ikv_pages_fork(self.shape, p.cache(0, granted=True), self.pages, len(src), i32(src), i32(dst), p.ema)
        per = d.rows // d.batch
        for s, t in zip(src, dst):
            n = int(d.len[s])
            for x in (d.len, d.next_pos, d.start):
                x[t] = x[s]
            for x in (d.pos, d.ema):
                x[t * per:(t + 1) * per] = x[s * per:(s + 1) * per]
            d.vnorm[:, t] = d.vnorm[:, s]
            for layer in range(d.layers):
                for g in range(d.kv_heads):
                    for pool in (d.k, d.v):
                        d.scatter(pool, t, layer, g, d.gather(pool, s, layer, g, n))

    def end(self, seqs):
        for c in self.both():
            c.len[seqs] = 0
        ikv.ikv_pages_release(self.shape, self.p.cache(0, granted=True), self.pages, 0)

    def rows(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda").to(self.p.torch_dtype)

    def same(self):
        p, d = self.both()
        assert ikv.ikv_device_status() == 0
        assert torch.equal(p.len, d.len) and torch.equal(p.next_pos, d.next_pos) and torch.equal(p.start, d.start)
        per = d.rows // d.batch
        for b, n in enumerate(d.len.tolist()):
            r = slice(b * per, (b + 1) * per)
            assert torch.equal(p.pos[r, :n], d.pos[r, :n]) and torch.equal(p.ema[r, :n], d.ema[r, :n])
            assert torch.equal(p.vnorm[:, b, :, :n], d.vnorm[:, b, :, :n])
            for layer in range(d.layers):
                for g in range(d.kv_heads):
                    for x, y in ((p.k, d.k), (p.v, d.v)):
                        assert torch.equal(p.gather(x, b, layer, g, n), d.gather(y, b, layer, g, n))
        held = (p.block_table > 0).sum()
        assert int(p.refs.sum()) == 1 + int(held) and int(p.refs.min()) == 0


SHAPES = [(5, 2, 4, 128, ikv.IKV_BF16, 16, 0), (5, 1, 7, 128, ikv.IKV_BF16, 64, 1), (5, 2, 2, 64, ikv.IKV_F32, 7, 0),
          (5, 3, 1, 64, ikv.IKV_BF16, 16, 1)]


def decode(pair, t, score=True, **kw):
    """ikv_step for all: every slot that it may write, 0 .. len, is made the sequence's own first."""
    p, d = pair.both()
    pair.writable(torch.zeros_like(p.len), p.len + 1)
    q = pair.rows(p.layers, p.batch, p.q_heads, p.head_dim)
    k, v = pair.rows(p.layers, p.batch, p.kv_heads, p.head_dim), pair.rows(p.layers, p.batch, p.kv_heads, p.head_dim)
    outs = []
    for c in pair.both():
        out = torch.full_like(q, 3.0)
        ws = c.step_workspace()
        ikv.ikv_step(c.shape(), c.params(0.8, refresh_period=1 if score else 2, **kw), c.cache(c.cap - 24), c.ema, t, q, k, v,
                     out, ws, ws.numel())
        outs.append(out)
    assert torch.equal(*outs)
    pair.same()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("mode,holes", [(ikv.IKV_COMPACT_STABLE, 0), (ikv.IKV_COMPACT_STABLE_SHORT, 0), (ikv.IKV_COMPACT_HOLEFILL, 0),
                                        (ikv.IKV_COMPACT_STABLE, 4), (ikv.IKV_COMPACT_STABLE_SHORT, 3), (ikv.IKV_COMPACT_HOLEFILL, 5)])
def test_steps_over_shared_pages(shape, mode, holes):
    """Prompts, forks, steps that evict at once or leave holes for a while, forks of what they left, ends."""
    rng = random.Random(holes)
    pair = Pair(*shape)
    for c in pair.both():
        c.budget.copy_(i32([50, 33, 50, 20, 50]))
    pair.prompt([70, 33, 0, 9, 0])
    pair.fork([0, 1], [2, 4])
    assert int((pair.p.refs[1:] > 1).sum()) > 0
    pair.same()
    for t in range(1, 9):
        decode(pair, t, score=rng.random() < 0.7, compact_mode=mode, max_holes=holes)
    pair.end([2, 3])
    pair.fork([4, 0], [2, 3])
    pair.same()
    for t in range(9, 20):
        decode(pair, t, compact_mode=mode, max_holes=holes)
    pair.end([0, 1, 2, 3, 4])
    assert pair.p.refs.tolist() == [1] + [0] * (pair.p.num_pages - 1)


@pytest.mark.parametrize("shape", SHAPES)
def test_appends_and_attention_over_shared_pages(shape):
    """Samples that only grow keep their prompt's pages shared: a page for the new token, attention and
    scores over all, and now and then an eviction into fresh pages."""
    pair = Pair(*shape)
    p, d = pair.both()
    for c in pair.both():
        c.budget.fill_(60)
    pair.prompt([75, 31, 0, 0, 0])
    pair.fork([0, 0, 1], [2, 3, 4])
    for t in range(26):
        pair.writable(None, torch.ones_like(p.len))
        x, y = pair.rows(p.layers, p.batch, p.kv_heads, p.head_dim), pair.rows(p.layers, p.batch, p.kv_heads, p.head_dim)
        q = pair.rows(p.batch, p.q_heads, p.head_dim)
        outs = []
        for c in pair.both():
            ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
            cache = c.cache(c.cap - 30, granted=c is p)
            ikv.ikv_append_token(c.shape(), cache, x, y, c.ema, t % 2, ws, ws.numel())
            n = ikv.ikv_attend_workspace_size(c.shape(), cache)
            ws, out = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros_like(q)
            for layer in range(c.layers):
                ikv.ikv_decode_attend_score(c.shape(), cache, layer, q, out, None, c.ema, 0.8, ws, n)
                outs.append(out.clone())
        pair.same()
        assert all(torch.equal(a, b) for a, b in zip(outs[:len(outs) // 2], outs[len(outs) // 2:]))
        if t == 3:
            assert int((p.refs[1:] > 1).sum()) > 0  # what lies in front of the samples' own tokens
        if t % 10 == 9:
            for c in pair.both():
                keep, n = torch.zeros(c.rows, c.cap, dtype=torch.int32, device="cuda"), torch.zeros(c.rows, dtype=torch.int32, device="cuda")
                ikv.ikv_select_budget(c.rows, c.cap, c.ema, c.len, c.rows_per_seq, c.budget, None, keep, n)
                if c is p:
                    ikv.ikv_pages_compact(c.shape(), c.cache(0, granted=True), pair.pages, keep, n, c.ema, pair.lacking, pair.ws, pair.ws.numel())
                    assert int(pair.lacking) == 0
                else:
                    ws = torch.zeros(ikv.ikv_compact_workspace_size(c.shape(), c.cache(0), ikv.IKV_COMPACT_STABLE), dtype=torch.uint8, device="cuda")
                    ikv.ikv_compact_kv(c.shape(), c.cache(c.cap), keep, n, c.ema, ikv.IKV_COMPACT_STABLE, ws, ws.numel())
            pair.same()
