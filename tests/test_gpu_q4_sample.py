"""The sampling example in lock-step with plain fp64: prompts stored in 4 bits, cut to their budget,
forked, continued, cut again, ended.

The reference keeps every sequence's rows as the values that the definition of the format gives
them, so what differs is rounding alone: outputs are bf16 (2^-8 of their size) of fp32 sums over
weights rounded to fp16 (2^-10 of the sum of their magnitudes, which is at most 6 / 0.5 as
large as a typical row, and shrinks with the number of rows: 2e-2 absolute covers both for outputs of
order one); utilities are fp32 sums of probabilities (1e-5).  A set kept by the cache is
right if no token outside it has a utility 1e-5 above one inside."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from sample_q4 import Model, Sampler  # noqa: E402
from test_gpu_q4 import quantise, values  # noqa: E402

from paper_2609_03515_gb300 import ikv  # noqa: E402

pytestmark = pytest.mark.gpu


class Plain:
    """One sequence: rows by layer, positions, utility."""

    def __init__(self, layers):
        self.k, self.v = [None] * layers, [None] * layers
        self.pos, self.m = [], None

    def copy(self):
        p = Plain(len(self.k))
        p.k, p.v, p.pos, p.m = list(self.k), list(self.v), list(self.pos), self.m.clone()
        return p


def stored(x):
    return values(*quantise(x))  # [n, kv_heads, d] fp64


def plain_step(model, p, x, alpha):
    """x [1, hidden] of the GPU's own input to each layer is passed in by layer: returns outputs by layer."""
    outs = []
    p.m = torch.cat([p.m, torch.zeros(1, dtype=torch.float64, device="cuda")])
    for layer in range(model.layers):
        q, k, v = model.qkv(layer, x[layer])
        p.k[layer] = torch.cat([p.k[layer], stored(k)])
        p.v[layer] = torch.cat([p.v[layer], stored(v)])
        G = model.q_heads // model.kv_heads
        kk = p.k[layer].repeat_interleave(G, 1)
        vv = p.v[layer].repeat_interleave(G, 1)
        z = torch.einsum("hd,nhd->hn", q[0].double(), kk) / math.sqrt(model.head_dim)
        a = torch.softmax(z, -1)
        outs.append(torch.einsum("hn,nhd->hd", a, vv))
        p.m = alpha * p.m + (1 - alpha) * a.mean(0)
    return outs


def test_sampling_follows_the_plain_computation():
    model = Model(layers=3, hidden=96, q_heads=8, kv_heads=2, head_dim=64, seed=4)
    gen = torch.Generator(device="cuda").manual_seed(9)
    batch, budget, every = 5, 40, 12
    s = Sampler(model, batch, budget, 300, pool_pages=90, every=every, page_size=16)
    plain = [None] * batch
    for b, n in ((0, 201), (3, 77)):
        x = torch.randn(n, model.hidden, generator=gen, device="cuda")
        s.prompt(b, x)
        p = plain[b] = Plain(model.layers)
        for layer in range(model.layers):
            _, k, v = model.qkv(layer, x)
            p.k[layer], p.v[layer] = stored(k), stored(v)
        p.pos, p.m = list(range(n)), torch.zeros(n, dtype=torch.float64, device="cuda")
    full = s.pages_in_use()
    assert full == -(-201 // 16) + -(-77 // 16)
    nxt = {0: 201, 3: 77}
    forked = False
    x = torch.randn(batch, model.hidden, generator=gen, device="cuda")
    seen = []
    after = model.after
    model.after = lambda layer, h, out: (seen.append((h.clone(), out.clone())), after(layer, h, out))[1]
    for t in range(1, 30):
        seen.clear()
        cut = t == 1 or t % every == 0
        x = s.step(x, cut=t == 1)
        c = s.c
        for b in range(batch):
            p = plain[b]
            if p is None:
                assert int(c.len[b]) == 0
                continue
            outs = plain_step(model, p, [h[b:b + 1] for h, _ in seen], s.alpha)
            for (_, out), want in zip(seen, outs):
                assert float((out[b].double() - want).abs().max()) < 2e-2, (t, b)
            p.pos.append(nxt[b])
            nxt[b] += 1
            n = int(c.len[b])
            got = c.pos[b, :n].tolist()
            if cut and len(p.pos) > budget:
                assert n == budget and got == sorted(got) and set(got) <= set(p.pos)
                inside = torch.tensor([q in set(got) for q in p.pos], device="cuda")
                assert float(p.m[inside].min()) >= float(p.m[~inside].max()) - 1e-5
                at = inside.nonzero()[:, 0]
                p.pos, p.m = got, p.m[at]
                p.k, p.v = [k[at] for k in p.k], [v[at] for v in p.v]
            assert got == p.pos
            assert float((c.ema[b, :n].double() - p.m).abs().max()) < 1e-5, (t, b)
        if t == 1:
            assert s.pages_in_use() == 2 * -(-budget // 16) < full
        if t == 3 and not forked:
            before = s.pages_in_use()
            s.fork([0, 0, 3], [1, 2, 4])
            assert s.pages_in_use() == before
            for a, b in ((0, 1), (0, 2), (3, 4)):
                plain[b], nxt[b] = plain[a].copy(), nxt[a]
            forked = True
            x = x[[0, 0, 0, 3, 3]] + 0.5 * torch.randn(batch, model.hidden, generator=gen, device="cuda")
        if t == 20:
            s.end([1, 3])
            plain[1] = plain[3] = None
    assert ikv.ikv_device_status() == 0
    s.end(list(range(batch)))
    assert s.pages_in_use() == 0 and s.c.refs.tolist() == [1] + [0] * 90
