"""Several continuations of each prompt, from one cache held in 4 bits whose pages they share.

    python examples/sample_q4.py [--prompt 2000 --samples 8 --steps 96 --budget 256]

The calls of include/ikv.h in the order a server makes them:
  prompt   ikv_pages_writable (pages for its slots), ikv_q4_store layer by layer;
  first    one step scores the whole prompt, ikv_select_budget keeps its budget of tokens and
           ikv_pages_compact gives the other pages back;
  fork     ikv_pages_fork: the samples share the prompt's pages;
  step     ikv_pages_writable (a new page, or a copy of a shared one), ikv_q4_append_token for
           the books, then in each layer ikv_q4_store and ikv_q4_attend_score, which folds
           the layer's score into the utility; every `every` steps the cache is cut back;
  end      ikv_pages_release.
A pool that runs short loses nothing: ikv_q4_append_token and ikv_q4_store leave out a sequence whose
slots ikv_pages_writable did not grant, and the loop finds the error bit at its next cut.
The model is a stand-in of random weights: a layer projects its input to q, k and v and adds the
attention's output back.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_03515_gb300 import Q4Cache, ikv  # noqa: E402


class Model:
    def __init__(self, layers=4, hidden=256, q_heads=8, kv_heads=2, head_dim=64, seed=0):
        self.layers, self.hidden = layers, hidden
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, m):
            return torch.randn(layers, n, m, generator=gen, device="cuda") * n ** -0.5

        self.wq, self.wk = 3.0 * weight(hidden, q_heads * head_dim), weight(hidden, kv_heads * head_dim)
        self.wv, self.wo = weight(hidden, kv_heads * head_dim), weight(q_heads * head_dim, hidden)

    def qkv(self, layer, x):
        """bf16 q [n, q_heads, d], k and v [n, kv_heads, d] of inputs x [n, hidden]."""
        n, d = x.shape[0], self.head_dim
        return ((x @ self.wq[layer]).to(torch.bfloat16).view(n, self.q_heads, d),
                (x @ self.wk[layer]).to(torch.bfloat16).view(n, self.kv_heads, d),
                (x @ self.wv[layer]).to(torch.bfloat16).view(n, self.kv_heads, d))

    def after(self, layer, x, out):
        return torch.tanh(x + out.float().flatten(1) @ self.wo[layer])


class Sampler:
    """The cache of `batch` sequences with `pool_pages` pages, and what a decode loop does with it."""

    def __init__(self, model, batch, budget, cap_tokens, pool_pages, every=32, alpha=0.9, page_size=16):
        m = self.model = model
        self.batch, self.budget, self.every, self.alpha = batch, budget, every, alpha
        c = self.c = Q4Cache(batch, m.layers, m.q_heads, m.kv_heads, m.head_dim, cap_tokens, page_size=page_size,
                             pool_pages=pool_pages)
        c.budget.fill_(budget)
        i32 = {"dtype": torch.int32, "device": "cuda"}
        self.slot = torch.full((batch,), -1, **i32)
        self.lacking = torch.zeros(1, **i32)
        self.keep, self.keep_len = torch.zeros(c.rows, c.cap, **i32), torch.zeros(c.rows, **i32)
        self.shape, self.q4, self.pages = c.shape(), c.q4(), c.pages()
        self.cache = c.cache(c.cap - 1)
        self.ws, self.pages_ws = c.attend_workspace(), c.pages_workspace()
        self.out = torch.zeros(batch, m.q_heads, m.head_dim, dtype=torch.bfloat16, device="cuda")
        self.t = 0

    def prompt(self, b, x):
        """Sequence b's prompt: x [tokens, hidden].  (A layer's K and V come from the inputs here; a
        model's come from the layer before.)"""
        c, n = self.c, x.shape[0]
        only = torch.full((self.batch,), -1, dtype=torch.int32, device="cuda")
        only[b] = 0
        ikv.ikv_pages_writable(self.shape, self.cache, self.pages, only, None, n, self.lacking, self.pages_ws,
                               self.pages_ws.numel())
        if int(self.lacking):
            raise RuntimeError("the prompt needs %d more pages than are free" % int(self.lacking))
        for layer in range(self.model.layers):
            _, k, v = self.model.qkv(layer, x)
            rows = ikv.ikv_rows(0, 0, k.stride(0), k.stride(1), None)
            ikv.ikv_q4_store(self.shape, self.cache, self.q4, layer, 1, k, v, rows, only, None, n)
        c.len[b] = n
        c.next_pos[b] = n
        c.pos[b, :n] = torch.arange(n, dtype=torch.int32, device="cuda")
        c.ema[b, :n] = 0.0

    def fork(self, src, dst):
        i32 = {"dtype": torch.int32, "device": "cuda"}
        ikv.ikv_pages_fork(self.shape, self.cache, self.pages, len(src), torch.tensor(src, **i32),
                           torch.tensor(dst, **i32), self.c.ema)

    def step(self, x, cut=False):
        """One token of every sequence that holds any: inputs x [batch, hidden] -> the last layer's output."""
        c, m = self.c, self.model
        live = c.len > 0
        first = torch.where(live, c.len, -1)
        ikv.ikv_pages_writable(self.shape, self.cache, self.pages, first, None, 1, None, self.pages_ws,
                               self.pages_ws.numel())
        # (sequences without a prompt were granted nothing and stay empty)
        ikv.ikv_q4_append_token(self.shape, self.cache, self.q4, None, None, c.ema, 0, self.slot)
        for layer in range(m.layers):
            q, k, v = m.qkv(layer, x)
            rows = ikv.ikv_rows(0, k.stride(0), k.stride(0), k.stride(1), None)
            ikv.ikv_q4_store(self.shape, self.cache, self.q4, layer, 1, k, v, rows, self.slot, None, 1)
            ikv.ikv_q4_attend_score(self.shape, self.cache, self.q4, layer, q, self.out, None, c.ema, self.alpha, self.ws,
                                    self.ws.numel())
            x = m.after(layer, x, self.out)
        self.t += 1
        if cut or self.t % self.every == 0:
            status = ikv.ikv_device_status()
            if status:
                raise RuntimeError("tokens were left out: device status %d" % status)
            ikv.ikv_select_budget(c.rows, c.cap, c.ema, c.len, 1, c.budget, None, self.keep, self.keep_len)
            ikv.ikv_pages_compact(self.shape, self.cache, self.pages, self.keep, self.keep_len, c.ema, None, self.pages_ws,
                                  self.pages_ws.numel())
        return x

    def end(self, seqs):
        self.c.len[seqs] = 0
        ikv.ikv_pages_release(self.shape, self.cache, self.pages, 0)

    def pages_in_use(self):
        return int((self.c.refs[1:] > 0).sum())


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompt", type=int, default=2000)
    ap.add_argument("--samples", type=int, default=8)
    ap.add_argument("--steps", type=int, default=96)
    ap.add_argument("--budget", type=int, default=256)
    a = ap.parse_args()
    model = Model()
    ps = 16
    cap = max(a.prompt, a.budget) + 64
    s = Sampler(model, a.samples, a.budget, cap, pool_pages=(a.prompt + 2 * a.samples * (a.budget + 64)) // ps + 8, page_size=ps)
    gen = torch.Generator(device="cuda").manual_seed(1)
    s.prompt(0, torch.randn(a.prompt, model.hidden, generator=gen, device="cuda"))
    print("prompt of %d tokens: %d pages" % (a.prompt, s.pages_in_use()))
    x = torch.randn(1, model.hidden, generator=gen, device="cuda").repeat(a.samples, 1)
    x = s.step(x, cut=True)
    print("cut to %d tokens:    %d pages" % (int(s.c.len[0]), s.pages_in_use()))
    s.fork([0] * (a.samples - 1), list(range(1, a.samples)))
    print("%d samples:           %d pages" % (a.samples, s.pages_in_use()))
    x = x[:1] + 0.3 * torch.randn(a.samples, model.hidden, generator=gen, device="cuda")  # they part here
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        x = s.step(x)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print("%d steps later:      %d pages, %.0f tokens/s" % (a.steps, s.pages_in_use(), a.steps * a.samples / t))
    s.end(list(range(a.samples)))
    print("ended:               %d pages, device status %d" % (s.pages_in_use(), ikv.ikv_device_status()))


if __name__ == "__main__":
    main()
