"""Caches for the shared-prefix and sliding-window attentions, and both in 64 bits.

Everything outside the sequences' live rows is NaN: the rest of the pools, the rows of dead slots, the
outputs' and scores' other places are checked to stay as they were."""
import math

import torch

from paper_2609_03515_gb300 import ikv

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
MARK = 77.0  # what buffers hold before a call


class Cache:
    def __init__(self, lens, kv_heads, group, d, dtype, page, seed, starts=None, dead=0.0, gran="seq", layers=2,
                 spread=1.0, extra_pages=1, share=()):
        """share: (leader, others, slots) whose first slots hold the same rows"""
        g = torch.Generator().manual_seed(seed)
        self.lens, self.g, self.G, self.d, self.dtype, self.page = list(lens), kv_heads, group, d, dtype, page
        nb = len(lens)
        self.starts = list(starts) if starts else [0] * nb
        self.gran, self.layers, self.dead = gran, layers, dead
        self.h = kv_heads * group
        held = [(s + n + page - 1) // page for s, n in zip(self.starts, lens)]
        self.max_pages = max(held) + extra_pages
        self.cap = self.max_pages * page
        self.pages = sum(held) + 2
        ids = 1 + torch.randperm(self.pages - 1, generator=g)
        self.table = torch.zeros(nb, self.max_pages, dtype=torch.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = ids[at:at + n].int()
            at += n
        # rows in 64 bits of what the cache holds: [nb][layers][kv][len][d]
        self.k, self.v = [], []
        for b in range(nb):
            self.k.append(torch.randn(layers, kv_heads, lens[b], d, generator=g).mul_(spread).to(DT[dtype]))
            self.v.append(torch.randn(layers, kv_heads, lens[b], d, generator=g).to(DT[dtype]))
        for lead, others, n in share:
            for b in others:
                self.k[b][:, :, :n] = self.k[lead][:, :, :n]
                self.v[b][:, :, :n] = self.v[lead][:, :, :n]
        rows = nb * kv_heads if gran == "kvhead" else nb
        self.pos = torch.arange(self.cap, dtype=torch.int32).repeat(rows, 1)
        if dead:
            self.pos[torch.rand(rows, self.cap, generator=g) < dead] = -1

    def alive(self, b, i):
        r = b * self.g + i if self.gran == "kvhead" else b
        return self.pos[r, :self.lens[b]] >= 0

    def device(self, hidden=math.nan):
        """Fills the pools: NaN (or `hidden`) wherever no sequence has a slot."""
        self.kp = torch.full((self.layers, self.pages, self.g, self.page, self.d), hidden, dtype=DT[self.dtype])
        self.vp = self.kp.clone()
        for b, n in enumerate(self.lens):
            at = torch.arange(n) + self.starts[b]
            p, o = self.table[b][at // self.page].long(), at % self.page
            self.kp[:, p, :, o] = self.k[b].permute(2, 0, 1, 3)
            self.vp[:, p, :, o] = self.v[b].permute(2, 0, 1, 3)
        self.t = {n: x.cuda() for n, x in (("k", self.kp), ("v", self.vp), ("table", self.table), ("pos", self.pos))}
        self.t["len"] = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.t["start"] = torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.t["next_pos"] = self.t["len"].clone()
        return self

    def shape(self):
        return ikv.ikv_shape(len(self.lens), self.layers, self.h, self.g, self.d,
                             ikv.IKV_F32 if self.dtype == "f32" else ikv.IKV_BF16,
                             ikv.IKV_GRAN_KVHEAD if self.gran == "kvhead" else ikv.IKV_GRAN_SEQ)

    def cache(self):
        t = {n: x.data_ptr() for n, x in self.t.items()}
        return ikv.ikv_cache(t["k"], t["v"], t["table"], self.pages, self.page, self.max_pages, t["len"], t["pos"],
                             t["next_pos"], max(self.lens), t["start"] if any(self.starts) else None,
                             1 if self.dead else 0, None, 0)


def attention(c, layer, b, i, q, seen, k=None, v=None):
    """In 64 bits: out [rows][d], weights [rows][slots], and bounds of the errors of a 32-bit evaluation
    (and of weights rounded to bf16) for queries q [rows][d] of sequence b and KV head i, seen [rows][slots].

    A product q . k of d terms, each rounded and added in 32 bits in any order, is off by at most
    (d + 1) 2^-24 sum |q k|; with the scale e_z = (d + 3) 2^-24 sum |q k| / sqrt(d).  A weight is then off
    by a factor 1 + 2 e_z (its own and the maximum's or the sum's), 2^-22 of exp2 and the products
    around it, of the sum of n and of a few parts' merges (n + 64) 2^-24."""
    k = (c.k[b][layer, i] if k is None else k).double()
    v = (c.v[b][layer, i] if v is None else v).double()
    q = q.double()
    z = q @ k.T / math.sqrt(c.d)
    z = torch.where(seen, z, torch.full_like(z, -math.inf))
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    s = e.sum(-1, keepdim=True)
    p = e / torch.where(s > 0, s, torch.ones_like(s))
    v0 = torch.where(seen.any(0)[:, None], v, torch.zeros_like(v))  # (rows nobody sees may be NaN)
    out = p @ v0
    eps = 2.0 ** -24
    mag = torch.where(seen, q.abs() @ torch.where(seen.any(0)[:, None], k, torch.zeros_like(k)).abs().T, 0.0)
    e_z = (c.d + 3) * eps * mag.amax(-1, keepdim=True) / math.sqrt(c.d)
    n = seen.shape[1]
    rel = 4 * e_z + 2.0 ** -21 + (n + 64) * eps  # of a weight
    tol = (p @ v0.abs()) * (rel + (n + 64) * eps + (2.0 ** -8 if c.dtype == "bf16" else 0.0))
    half = 2.0 ** -8 if c.dtype == "bf16" else eps
    return out, p, tol * (1 + half) + out.abs() * half + 1e-30, p * (rel + z.abs().nan_to_num(posinf=0.0) * 2.0 ** -22 + 2.0 ** -20)


def window_seen(n, count, i0, i1, window, sinks):
    p = torch.arange(n - count + i0, n - count + i1)[:, None]
    j = torch.arange(n)[None]
    near = (j > p - window) if window > 0 else torch.ones(1, 1, dtype=torch.bool)
    return (j <= p) & (near | (j < sinks))
