"""Several continuations of each prompt from a bf16 cache: the prompt is attended once in chunks, then its samples
decode over its pages together.

    python examples/sample_shared.py [--prompt 2000 --samples 8 --steps 96 --budget 128 --window 0 --sinks 4]

The calls of include/ikv.h in the order a server makes them:
  prompt   ikv_pages_writable (pages for its slots), then chunk by chunk and layer by layer the chunk's K and V
           into their slots and ikv_window_attend (--window 0: plain causal attention);
  fork     ikv_pages_fork: the samples share the prompt's pages;
  step     ikv_pages_writable (a new page, or a copy of a shared one), ikv_append_token for the books, then in
           each layer the token's K and V into its slot and ikv_prefix_attend_score, which reads the prompt once
           for all of its samples and folds the layer's score into the utility;
  cut      ikv_select_budget and ikv_pages_compact: each sample keeps the prompt and `budget` tokens of its own
           (the prompt's utility is infinite, so it stays shared);
  end      ikv_pages_release.
The model is the stand-in of sample_q4.py.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from sample_q4 import Model  # noqa: E402

from paper_2609_03515_gb300 import DecodeCache, ikv  # noqa: E402


class SharedSampler:
    """The cache of `batch` sequences with `pool_pages` pages, and what a decode loop does with it."""

    def __init__(self, model, batch, budget, cap_tokens, pool_pages, window=0, sinks=4, chunk=512, every=32, alpha=0.9,
                 page_size=16):
        m = self.model = model
        self.batch, self.budget, self.every, self.alpha, self.chunk = batch, budget, every, alpha, chunk
        self.sinks, self.width = sinks, window
        c = self.c = DecodeCache(batch, m.layers, m.q_heads, m.kv_heads, m.head_dim, cap_tokens, page_size=page_size,
                                 pool_pages=pool_pages)
        i32 = {"dtype": torch.int32, "device": "cuda"}
        self.lacking = torch.zeros(1, **i32)
        self.keep, self.keep_len = torch.zeros(c.rows, c.cap, **i32), torch.zeros(c.rows, **i32)
        self.shape, self.cache, self.pages = c.shape(), c.cache(c.cap - 1), c.pages()
        self.pages_ws = c.pages_workspace()
        self.out = torch.zeros(batch, m.q_heads, m.head_dim, dtype=torch.bfloat16, device="cuda")
        none = torch.zeros(m.layers, batch, m.kv_heads, m.head_dim, dtype=torch.bfloat16, device="cuda")
        self.no_rows = none  # (the rows follow layer by layer)
        self.append_ws = torch.empty((4 * batch + 255) // 256 * 256, dtype=torch.uint8, device="cuda")
        self.group([])
        self.t = 0

    def group(self, groups):
        """groups: (sequences, slots they share) of each; kept on the device for the steps."""
        self.prefix = self.c.prefix([g for g, _ in groups], [n for _, n in groups])
        self.prefix_ws = self.c.prefix_workspace(self.prefix)

    def put(self, layer, seqs, slots, k, v):
        """Rows k, v [n, kv_heads, d] into slots [n] of sequences [n]."""
        c = self.c
        page = c.block_table[seqs, slots // c.page_size].long()
        c.k[layer, page, :, slots % c.page_size] = k
        c.v[layer, page, :, slots % c.page_size] = v

    def prompt(self, b, x):
        """Sequence b's prompt: x [tokens, hidden].  Returns the last layer's output of its last token."""
        c, n = self.c, x.shape[0]
        only = torch.full((self.batch,), -1, dtype=torch.int32, device="cuda")
        only[b] = 0
        ikv.ikv_pages_writable(self.shape, self.cache, self.pages, only, None, n, self.lacking, self.pages_ws,
                               self.pages_ws.numel())
        if int(self.lacking):
            raise RuntimeError("the prompt needs %d more pages than are free" % int(self.lacking))
        last = None
        for a in range(0, n, self.chunk):
            h = x[a:a + self.chunk]
            slots = torch.arange(a, a + len(h), device="cuda")
            c.len[b] = a + len(h)
            counts = [len(h) if i == b else 0 for i in range(self.batch)]
            w = c.window(self.width, self.sinks, counts)
            ws = c.window_workspace(w)
            for layer in range(self.model.layers):
                q, k, v = self.model.qkv(layer, h)
                self.put(layer, torch.full_like(slots, b), slots, k, v)
                out = torch.empty_like(q)
                ikv.ikv_window_attend(self.shape, self.cache, w, layer, q, out, ws, ws.numel())
                h = self.model.after(layer, h, out)
            last = h[-1:]
        c.next_pos[b] = n
        c.pos[b, :n] = torch.arange(n, dtype=torch.int32, device="cuda")
        c.ema[b, :n] = math.inf  # the prompt is never cut
        c.budget[b] = n + self.budget
        return last

    def fork(self, src, dst):
        i32 = {"dtype": torch.int32, "device": "cuda"}
        ikv.ikv_pages_fork(self.shape, self.cache, self.pages, len(src), torch.tensor(src, **i32),
                           torch.tensor(dst, **i32), self.c.ema)
        self.c.budget[torch.tensor(dst, device="cuda")] = self.c.budget[torch.tensor(src, device="cuda")]

    def step(self, x):
        """One token of every sequence: inputs x [batch, hidden] -> the last layer's output."""
        c, m = self.c, self.model
        ikv.ikv_pages_writable(self.shape, self.cache, self.pages, None, None, 1, None, self.pages_ws,
                               self.pages_ws.numel())
        slots = c.len.long()
        ikv.ikv_append_token(self.shape, self.cache, self.no_rows, self.no_rows, c.ema, 0, self.append_ws,
                             self.append_ws.numel())
        seqs = torch.arange(self.batch, device="cuda")
        for layer in range(m.layers):
            q, k, v = m.qkv(layer, x)
            self.put(layer, seqs, slots, k, v)
            ikv.ikv_prefix_attend_score(self.shape, self.cache, self.prefix, layer, q, self.out, None, c.ema, self.alpha,
                                        self.prefix_ws, self.prefix_ws.numel())
            x = m.after(layer, x, self.out)
        self.t += 1
        if self.t % self.every == 0:
            status = ikv.ikv_device_status()
            if status:
                raise RuntimeError("device status %d" % status)
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
    ap.add_argument("--budget", type=int, default=128)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=4)
    a = ap.parse_args()
    model, ps = Model(), 16
    own = a.budget + 64
    s = SharedSampler(model, a.samples, a.budget, a.prompt + own, (a.prompt + a.samples * 2 * own) // ps + 8 * a.samples,
                      window=a.window, sinks=a.sinks, page_size=ps)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = s.prompt(0, torch.randn(a.prompt, model.hidden, generator=gen, device="cuda"))
    print("prompt of %d tokens: %d pages" % (a.prompt, s.pages_in_use()))
    s.fork([0] * (a.samples - 1), list(range(1, a.samples)))
    s.group([(list(range(a.samples)), a.prompt)])
    x = x + 0.3 * torch.randn(a.samples, model.hidden, generator=gen, device="cuda")  # they part here
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
