"""The shared-prompt example in lock-step with plain 64 bits: prompts attended in chunks through a window, forked,
continued together, cut, continued, ended.

Each layer's reference takes the q, k and v that the cache was given, so what differs is the attention alone: fp32
sums, weights rounded to bf16 (2^-8 of sum p |v|), outputs rounded to bf16 (2^-8).  Utilities are fp32 EMAs of
probabilities of at most 1, over at most a few dozen updates: 1e-5 absolute.  A kept set is right if no token
outside it has a utility 1e-5 above one inside."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import sample_shared  # noqa: E402
from sample_q4 import Model  # noqa: E402
from sample_shared import SharedSampler  # noqa: E402

from paper_2609_03515_gb300 import ikv  # noqa: E402

pytestmark = pytest.mark.gpu


class Recorder(Model):
    """The model, with what it was asked and told by layer."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.log = []

    def qkv(self, layer, x):
        t = super().qkv(layer, x)
        self.log.append([layer, *[y.clone() for y in t], None])
        return t

    def after(self, layer, x, out):
        self.log[-1][4] = out.clone()
        return super().after(layer, x, out)


def attend(q, k, v, seen):
    """q [n, H, d], k, v [m, g, d] in 64 bits, seen [n, m] -> out [n, H, d], weights [n, H, m], sum p |v|"""
    G = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    z = torch.einsum("nhd,mhd->nhm", q, k) / math.sqrt(q.shape[2])
    p = torch.softmax(torch.where(seen[:, None], z, torch.full_like(z, -math.inf)), -1)
    return torch.einsum("nhm,mhd->nhd", p, v), p, torch.einsum("nhm,mhd->nhd", p, v.abs())


def close(got, want, size):
    return bool(((got.double() - want).abs() <= 2.0 ** -8 * (want.abs() + size * 1.01) + 1e-6).all())


@pytest.mark.parametrize("head_dim,window,sinks", [(64, 0, 0), (128, 40, 3)])
def test_prompts_samples_cuts(head_dim, window, sinks):
    model = Recorder(layers=2, hidden=64, q_heads=8, kv_heads=2, head_dim=head_dim, seed=3)
    prompts, samples, budget = [150, 83], 3, 20
    batch = len(prompts) * samples
    s = SharedSampler(model, batch, budget, 256, 200, window=window, sinks=sinks, chunk=64, every=8, page_size=16)
    gen = torch.Generator(device="cuda").manual_seed(4)
    plain = [{"k": [[], []], "v": [[], []], "m": None} for _ in range(batch)]
    x = torch.zeros(batch, 64, device="cuda")
    for i, n in enumerate(prompts):
        model.log.clear()
        x[i] = s.prompt(i, torch.randn(n, 64, generator=gen, device="cuda"))
        for layer, q, k, v, out in model.log:
            kk, vv = plain[i]["k"][layer], plain[i]["v"][layer]
            kk.append(k.double())
            vv.append(v.double())
            kall, vall = torch.cat(kk), torch.cat(vv)
            m, c = len(kall), len(q)
            p = torch.arange(m - c, m, device="cuda")[:, None]
            j = torch.arange(m, device="cuda")[None]
            seen = (j <= p) & ((j > p - window) | (j < sinks) if window else j >= 0)
            want, _, size = attend(q.double(), kall, vall, seen)
            assert close(out, want, size)
        plain[i]["m"] = torch.full((n,), math.inf, dtype=torch.float64, device="cuda")
    for i in range(len(prompts)):
        dst = [len(prompts) + i * (samples - 1) + k for k in range(samples - 1)]
        s.fork([i] * len(dst), dst)
        x[dst] = x[i].clone()
        for b in dst:
            plain[b] = {"k": [list(t) for t in plain[i]["k"]], "v": [list(t) for t in plain[i]["v"]],
                        "m": plain[i]["m"].clone()}
    groups = [[i] + [len(prompts) + i * (samples - 1) + k for k in range(samples - 1)] for i in range(len(prompts))]
    s.group(list(zip(groups, prompts)))
    pages = s.pages_in_use()
    assert pages == sum((n + 15) // 16 for n in prompts)  # shared, not copied
    x = x + 0.3 * torch.randn(batch, 64, generator=gen, device="cuda")
    lens = [prompts[g] for b in range(batch) for g in range(len(groups)) if b in groups[g]]
    for t in range(1, 41):
        model.log.clear()
        x = s.step(x)
        for b in range(batch):
            plain[b]["m"] = torch.cat([plain[b]["m"], torch.zeros(1, dtype=torch.float64, device="cuda")])
        for layer, q, k, v, out in model.log:
            for b in range(batch):
                pl = plain[b]
                pl["k"][layer].append(k[b:b + 1].double())
                pl["v"][layer].append(v[b:b + 1].double())
                kall, vall = torch.cat(pl["k"][layer]), torch.cat(pl["v"][layer])
                seen = torch.ones(1, len(kall), dtype=torch.bool, device="cuda")
                want, p, size = attend(q[b:b + 1].double(), kall, vall, seen)
                assert close(out[b:b + 1], want, size), (t, layer, b)
                pl["m"] = s.alpha * pl["m"] + (1 - s.alpha) * p[0].mean(0)
        for b in range(batch):
            pl = plain[b]
            n = len(pl["m"])
            if t % s.every == 0 and n > lens[b] + budget:
                keep = s.keep[b, :int(s.keep_len[b])].long()
                assert len(keep) == lens[b] + budget and bool((keep[:lens[b]].cpu() == torch.arange(lens[b])).all())
                gone = torch.ones(n, dtype=torch.bool, device="cuda")
                gone[keep] = False
                assert pl["m"][gone].max() <= pl["m"][keep].min() + 1e-5
                pl["m"] = pl["m"][keep]
                for name in ("k", "v"):
                    pl[name] = [[torch.cat(rows)[keep]] for rows in pl[name]]
            n = len(pl["m"])
            assert int(s.c.len[b]) == n
            own = s.c.ema[b, lens[b]:n].double()
            assert bool(((own - pl["m"][lens[b]:]).abs() <= 1e-5).all())
            assert bool(torch.isinf(s.c.ema[b, :lens[b]]).all())
    assert ikv.ikv_device_status() == 0
    # the prompts' whole pages are still shared
    shared = [int(s.c.refs[int(s.c.block_table[groups[i][0], 0])]) for i in range(len(prompts))]
    assert shared == [samples] * len(prompts)
    s.end(list(range(batch)))
    assert s.pages_in_use() == 0


def test_the_example_runs(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["sample_shared.py", "--prompt", "300", "--samples", "3", "--steps", "40", "--budget", "16",
                                      "--window", "100"])
    sample_shared.main()
    assert "ended:               0 pages, device status 0" in capsys.readouterr().out
