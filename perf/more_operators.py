"""Attention over a shared prefix and through a sliding window, as cases that can be timed and compared.

A case is one of two kinds:
  prefix   ikv_prefix_attend_score: one layer's decode attention of a batch whose sequences fall
           into groups with a common prefix, with or without the score of their tokens;
  window   ikv_window_attend: one layer's causal attention of the newest tokens of every sequence
           over its paged cache, through a window of the latest slots and the first few (sinks),
           from a single token a sequence to a whole prompt.  Window 0: every slot up to its own.

The plain forms below compute the same from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _prefix(name, **kw):
    c = {"name": name, "kind": "prefix", "groups": 1, "members": 4, "members_lo": 4, "alone": 0, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "page": 64, "plen_lo": 900, "plen_hi": 900, "tail_lo": 1,
         "tail_hi": 1, "gran": "seq", "score": False, "dead": 0.0, "start": 0}
    c.update(kw)
    return c


def _window(name, **kw):
    c = {"name": name, "kind": "window", "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16",
         "page": 64, "len_lo": 4096, "len_hi": 4096, "count_lo": 1, "count_hi": 1, "window": 1024, "sinks": 4,
         "gran": "seq", "dead": 0.0, "start": 0}
    c.update(kw)
    return c


def listed():
    return [
        # four samples of a short prompt, the Llama-3.1-8B shape: where latency counts
        _prefix("prefix_4_of_900", tail_lo=3, tail_hi=40),
        # sixteen samples of each of two 8k prompts, between two refreshes
        _prefix("prefix_2x16_of_8k", groups=2, members=16, members_lo=16, plen_lo=7777, plen_hi=8192, tail_lo=100,
                tail_hi=1200),
        # the same on a refresh step: the tokens' scores too
        _prefix("prefix_2x16_of_8k_score", groups=2, members=16, members_lo=16, plen_lo=7777, plen_hi=8192,
                tail_lo=100, tail_hi=1200, score=True),
        # the largest of its kind: the Qwen-2.5-7B shape (group of 7), 48 answers drawn from one 32k document
        _prefix("prefix_qwen_48_of_32k", members=48, members_lo=48, q_heads=28, kv_heads=4, page=128, plen_lo=32768,
                plen_hi=32768, tail_lo=64, tail_hi=2048),
        # small pages, groups of several sizes beside sequences that share nothing, evicted tokens
        # still in place, sequences that start inside a page, a utility row for each KV head
        _prefix("prefix_ragged_score", groups=5, members=7, members_lo=2, alone=6, page=16, plen_lo=600, plen_hi=4000,
                tail_lo=1, tail_hi=700, gran="kvhead", score=True, dead=0.03, start=21),
        # 32-bit queries and caches (accuracy studies), heads of 64
        _prefix("prefix_f32_d64", groups=2, members=4, members_lo=3, q_heads=16, kv_heads=4, head_dim=64, dtype="f32",
                page=16, plen_lo=1500, plen_hi=2000, tail_lo=10, tail_hi=300, score=True),
        # single-stream decode through a short window
        _window("window_b1_1k"),
        # batched decode with ragged lengths, a 4k window
        _window("window_b32_4k", batch=32, q_heads=28, kv_heads=4, page=128, len_lo=2000, len_hi=16384, window=4096),
        # a prompt of 8k through a window of 2k
        _window("window_prompt_8k", len_lo=8192, len_hi=8192, count_lo=8192, count_hi=8192, window=2048),
        # the largest: a whole prompt of 16k, every earlier slot visible
        _window("causal_prompt_16k", len_lo=16384, len_hi=16384, count_lo=16384, count_hi=16384, window=0, sinks=0),
        # chunks of several prompts behind what is cached of them, small pages, starts inside a page
        _window("window_chunks", batch=6, page=16, len_lo=700, len_hi=9000, count_lo=77, count_hi=1024, window=3000,
                sinks=16, start=21),
        # short ragged prompts in 32 bits, heads of 64
        _window("window_f32_d64", batch=8, q_heads=16, kv_heads=4, head_dim=64, dtype="f32", page=16, len_lo=17,
                len_hi=1021, count_lo=17, count_hi=1021, window=256),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"bf16": {"prefix": (1.6e8, 2.2e10), "window": (3.2e8, 6.0e11)},
            "f32": {"prefix": (1.5e8, 3.0e9), "window": (1.5e8, 1.5e10)}}
    while True:
        c = _draw(rng)
        by, fl = most[c["dtype"]][c["kind"]]
        w = work(c)
        if w["bytes"] <= by and w["flops"] <= fl and _held(c) <= 4.0e9:
            return c


def _held(c):
    """Bytes of the plain form's 32-bit K and V, roughly."""
    n = c["groups"] * c["members"] + c["alone"] if c["kind"] == "prefix" else c["batch"]
    longest = c["plen_hi"] + c["tail_hi"] if c["kind"] == "prefix" else c["len_hi"]
    return n * longest * c["kv_heads"] * c["head_dim"] * 8


def _draw(rng):
    shape = {"kv_heads": rng.choice([1, 2, 4, 8]), "head_dim": rng.choice([128, 128, 128, 64]),
             "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "page": rng.choice([16, 20, 48, 64, 128]),
             "gran": rng.choice(["seq", "kvhead"]), "dead": rng.choice([0.0, 0.0, 0.03, 0.5]),
             "start": rng.choice([0, 0, 5, 77])}
    shape["q_heads"] = shape["kv_heads"] * rng.choice([1, 2, 4, 4, 7, 8])
    if rng.random() < 0.5:
        members, hi, tail = _logint(rng, 2, 64), _logint(rng, 1, 33000), _logint(rng, 1, 2500)
        c = _prefix("", groups=rng.choice([1, 1, 2, 3, 6]), members=members,
                    members_lo=max(1, int(members * rng.choice([0.3, 1.0]))), alone=rng.choice([0, 0, 1, 5]),
                    plen_hi=hi, plen_lo=max(1, int(hi * rng.choice([0.2, 1.0]))), tail_hi=tail,
                    tail_lo=max(1, int(tail * rng.choice([0.05, 1.0]))), score=rng.random() < 0.5, **shape)
    else:
        hi = _logint(rng, 1, 33000)
        count = min(hi, rng.choice([1, 1, _logint(rng, 2, 16), _logint(rng, 1, 8192)]))
        c = _window("", batch=_logint(rng, 1, 48), len_hi=hi, len_lo=max(1, int(hi * rng.choice([0.1, 0.6, 1.0]))),
                    count_hi=count, count_lo=max(1, int(count * rng.choice([0.1, 1.0]))),
                    window=rng.choice([0, _logint(rng, 1, 8192), _logint(rng, 64, 8192)]),
                    sinks=rng.choice([0, 1, 4, 4, 130]), **shape)
    del c["name"]
    return c


# ---------------------------------------------------------------- sizes
def _spread(lo, hi, n):
    """n sizes over [lo, hi], ragged and fixed by the sizes alone."""
    if lo == hi or n == 1:
        return [hi] * n
    return [lo + (hi - lo) * ((i * 7919 + 3) % 997) // 996 for i in range(n)]


def _groups(case):
    """The sequences of each group: the prompts first, then the samples of each, then those alone."""
    sizes = _spread(case["members_lo"], case["members"], case["groups"])
    at, groups = case["groups"], []
    for i, n in enumerate(sizes):
        groups.append([i] + list(range(at, at + n - 1)))
        at += n - 1
    return groups, at + case["alone"]


def _plens(case):
    return _spread(case["plen_lo"], case["plen_hi"], case["groups"])


def _lens(case):
    if case["kind"] == "window":
        return _spread(case["len_lo"], case["len_hi"], case["batch"])
    groups, n = _groups(case)
    lens = _spread(case["tail_lo"], case["tail_hi"], n)
    for p, group in zip(_plens(case), groups):
        for b in group:
            lens[b] += p
    return lens


def _counts(case):
    counts = _spread(case["count_lo"], case["count_hi"], case["batch"])
    return [min(a, b) for a, b in zip(counts, _lens(case))]


def _starts(case, n):
    return [(case["start"] * (b + 1)) % 211 if case["start"] else 0 for b in range(n)]


def _visible(n, count, window, sinks):
    """Slots that some query of a sequence sees, and pairs of a query and a slot that it sees."""
    w = window if window > 0 else n
    first = max(0, n - count - w + 1)  # of the first query's window
    slots = n - first + min(sinks, first)
    lo = n - count + 1  # slots up to the first query's own
    full = max(0, n - max(lo, w) + 1)  # queries whose window is full
    part = count - full
    pairs = full * w + part * lo + part * (part - 1) // 2
    for k in range(sinks):  # sink k is seen apart by the queries at p >= k + w
        pairs += max(0, min(count, n - (k + w)))
    return slots, pairs


def work(case):
    d, g, h = case["head_dim"], case["kv_heads"], case["q_heads"]
    eb = 4 if case["dtype"] == "f32" else 2
    lens = _lens(case)
    if case["kind"] == "prefix":
        groups, n = _groups(case)
        plens = _plens(case)
        rows = sum(lens) - sum(p * (len(m) - 1) for p, m in zip(plens, groups))
        by = rows * g * 2 * d * eb + 2 * n * h * d * eb
        if case["score"]:
            by += 4 * sum(lens) * (g if case["gran"] == "kvhead" else 1)
        return {"bytes": by, "flops": 4 * sum(lens) * h * d}
    rows = pairs = 0
    for n, c in zip(lens, _counts(case)):
        a, b = _visible(n, c, case["window"], case["sinks"])
        rows += a
        pairs += b
    return {"bytes": rows * g * 2 * d * eb + 2 * sum(_counts(case)) * h * d * eb, "flops": 4 * pairs * h * d}


# ---------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _normal(shape, gen, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the descriptors and the workspace that a program keeps
        s["plan"] = _plan_prefix(s) if case["kind"] == "prefix" else _plan_window(s)
    return s


def run(state):
    if state["case"]["kind"] == "prefix":
        return _own_prefix(state) if own else _plain_prefix(state)
    return _own_window(state) if own else _plain_window(state)


def _pools(case, pages, gen):
    """Two layers of K and V, the second attended: keys around a direction of their head for one
    token in a hundred, the rest normal.  Returns the pools and the directions."""
    g, d, ps = case["kv_heads"], case["head_dim"], case["page"]
    u = torch.nn.functional.normalize(_normal((g, d), gen), dim=-1) * 8.0
    heavy = torch.rand(pages, ps, generator=gen, device="cuda") < 0.01
    pools = []
    for name in ("k", "v"):
        x = _normal((2, pages, g, ps, d), gen, DTYPES[case["dtype"]])
        if name == "k":
            at, off = torch.nonzero(heavy, as_tuple=True)
            x[:, at, :, off] = (3.0 * u + 0.3 * x[:, at, :, off].float()).to(x.dtype)
        pools.append(x)
    return pools[0], pools[1], u


def _inputs(case, seed):
    gen = _generator(seed)
    g, d, h, ps = case["kv_heads"], case["head_dim"], case["q_heads"], case["page"]
    lens = _lens(case)
    nb = len(lens)
    starts = _starts(case, nb)
    if case["kind"] == "prefix":
        groups, _ = _groups(case)
        for m in groups:  # a fork continues where its prompt starts
            for b in m:
                starts[b] = starts[m[0]]
    held = [(x + n + ps - 1) // ps for x, n in zip(starts, lens)]
    max_pages = max(held) + 1
    cap = max_pages * ps
    total = nb * max_pages if case["kind"] == "window" else sum(held) + 1
    ids = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    k, v, u = _pools(case, total, gen)
    table = torch.zeros(nb, max_pages, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(nb):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    for b in range(nb):  # the first four tokens draw attention
        slot = starts[b] + torch.arange(min(4, lens[b]), device="cuda")
        k[:, table[b, slot // ps].long(), :, slot % ps] *= 4.0
    s = {"case": case, "k": k, "v": v, "table": table, "len": _i32(lens), "start": _i32(starts) if case["start"] else None,
         "lens": lens, "starts": starts}
    rows = nb * g if case["gran"] == "kvhead" else nb
    s["pos"] = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(rows, 1)
    if case["dead"]:
        s["pos"][torch.rand(rows, cap, generator=gen, device="cuda") < case["dead"]] = -1
    s["next_pos"] = s["len"].clone()
    if case["kind"] == "prefix":
        for p, m in zip(_plens(case), groups):
            lead = m[0]
            full = (starts[lead] + p) // ps  # pages shared by all of them; the next was copied
            rest = (starts[lead] + p) % ps
            for b in m[1:]:
                table[b, :full] = table[lead, :full]
                if rest:
                    for t in (k, v):
                        t[:, int(table[b, full]), :, :rest] = t[:, int(table[lead, full]), :, :rest]
        s["first"] = _i32([sum(len(m) for m in groups[:i]) for i in range(len(groups) + 1)])
        s["member"] = _i32([b for m in groups for b in m])
        s["plen"] = _i32(_plens(case))
        w = u.repeat_interleave(h // g, 0)[None] + 0.5 * _normal((nb, h, d), gen)
        s["q"] = (8.0 * torch.nn.functional.normalize(w, dim=-1)).to(DTYPES[case["dtype"]])
        s["out"] = torch.zeros_like(s["q"])
        s["score"] = torch.zeros(rows, cap, device="cuda") if case["score"] else None
        return s
    s["counts"] = _counts(case)
    n = sum(s["counts"])
    s["row0s"] = [sum(s["counts"][:b]) for b in range(nb)]
    s["row0"], s["count"] = _i32(s["row0s"]), _i32(s["counts"])
    # the queries as they lie in the rows of a fused projection, q | k | v
    s["qkv"] = torch.zeros(n, (h + 2 * g) * d, dtype=DTYPES[case["dtype"]], device="cuda")
    for a in range(0, n, 4096):
        e = min(n, a + 4096)
        w = u.repeat_interleave(h // g, 0)[None] + 0.5 * _normal((e - a, h, d), gen)
        s["qkv"][a:e, :h * d] = (8.0 * torch.nn.functional.normalize(w, dim=-1)).flatten(1).to(s["qkv"].dtype)
    s["out"] = torch.zeros(n, h, d, dtype=s["qkv"].dtype, device="cuda")
    return s


def _shape_cache(s):
    from paper_2609_03515_gb300 import ikv

    case = s["case"]
    ptr = lambda x: x.data_ptr() if x is not None else None  # noqa: E731
    shape = ikv.ikv_shape(len(s["lens"]), 2, case["q_heads"], case["kv_heads"], case["head_dim"],
                          ikv.IKV_F32 if case["dtype"] == "f32" else ikv.IKV_BF16,
                          ikv.IKV_GRAN_KVHEAD if case["gran"] == "kvhead" else ikv.IKV_GRAN_SEQ)
    cache = ikv.ikv_cache(s["k"].data_ptr(), s["v"].data_ptr(), s["table"].data_ptr(), s["k"].shape[1], case["page"],
                          s["table"].shape[1], s["len"].data_ptr(), s["pos"].data_ptr(), s["next_pos"].data_ptr(),
                          max(s["lens"]), ptr(s["start"]), 1 if case["dead"] else 0, None, 0)
    return ikv, shape, cache


def _plan_prefix(s):
    ikv, shape, cache = _shape_cache(s)
    prefix = ikv.ikv_prefix(s["plen"].numel(), s["first"].data_ptr(), s["member"].data_ptr(), s["plen"].data_ptr())
    n = ikv.ikv_prefix_workspace_size(shape, cache, prefix)
    return {"ikv": ikv, "shape": shape, "cache": cache, "prefix": prefix, "n": n,
            "ws": torch.empty(n, dtype=torch.uint8, device="cuda")}


def _own_prefix(s):
    p = s["plan"]
    p["ikv"].ikv_prefix_attend_score(p["shape"], p["cache"], p["prefix"], 1, s["q"], s["out"], s["score"], None, 0.0,
                                     p["ws"], p["n"], torch.cuda.current_stream())
    return {"out": s["out"], "score": s["score"]} if s["score"] is not None else {"out": s["out"]}


def _plan_window(s):
    ikv, shape, cache = _shape_cache(s)
    case = s["case"]
    window = ikv.ikv_window(case["window"], case["sinks"], s["row0"].data_ptr(), s["count"].data_ptr(),
                            max(s["counts"]), s["qkv"].shape[1], 0)
    n = ikv.ikv_window_workspace_size(shape, cache, window)
    return {"ikv": ikv, "shape": shape, "cache": cache, "window": window, "n": n,
            "ws": torch.empty(n, dtype=torch.uint8, device="cuda")}


def _own_window(s):
    p = s["plan"]
    p["ikv"].ikv_window_attend(p["shape"], p["cache"], p["window"], 1, s["qkv"], s["out"], p["ws"], p["n"],
                               torch.cuda.current_stream())
    return {"out": s["out"]}


# ---------------------------------------------------------------- plainly
def _plain_softmax(z, live):
    z = torch.where(live, z, torch.full_like(z, -math.inf))
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    sums = e.sum(-1, keepdim=True)
    return e / torch.where(sums > 0, sums, torch.ones_like(sums))


def _plain_prefix(s):
    case = s["case"]
    h, g, d, ps = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    nb, n = len(s["lens"]), max(s["lens"])
    slot = torch.arange(n, device="cuda")[None].expand(nb, n)
    at = slot + s["start"][:, None] if s["start"] is not None else slot
    at = torch.minimum(at, torch.full_like(at, s["table"].shape[1] * ps - 1))
    page, off = torch.gather(s["table"], 1, at // ps).long(), at % ps
    k = s["k"][1][page, :, off].float()  # [b, n, g, d]
    live = (slot < s["len"][:, None])[:, None].expand(nb, g, n)
    if case["dead"]:
        live = live & (s["pos"].view(nb, -1, s["pos"].shape[1])[:, :, :n] >= 0)
    z = torch.matmul(s["q"].float().view(nb, g, h // g, d), k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    del k
    p = _plain_softmax(z, live[:, :, None])
    v = s["v"][1][page, :, off].float()
    v = torch.where(live.transpose(1, 2)[..., None], v, torch.zeros_like(v))
    s["out"].copy_(torch.matmul(p, v.transpose(1, 2)).reshape(nb, h, d))
    if s["score"] is None:
        return {"out": s["out"]}
    rows = s["score"].shape[0]
    pooled = p.mean(2).view(rows, n) if case["gran"] == "kvhead" else p.view(nb, h, n).mean(1)
    inside = (slot < s["len"][:, None]).repeat_interleave(rows // nb, 0)
    s["score"][:, :n] = torch.where(inside, pooled, s["score"][:, :n])
    return {"out": s["out"], "score": s["score"]}


def _plain_window(s):
    case = s["case"]
    h, g, d, ps = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    nb, most, longest = len(s["lens"]), max(s["counts"]), max(s["lens"])
    sinks = min(case["sinks"], longest)
    if most <= 16:  # all sequences at once, rows padded to the longest count
        blocks = [(list(range(nb)), 0, most)]
    else:
        blocks = [([b], a, min(1024, s["counts"][b] - a)) for b in range(nb) for a in range(0, s["counts"][b], 1024)]
    q_all = s["qkv"][:, :h * d].unflatten(1, (g, h // g, d))
    for seqs, a, nq in blocks:
        n = torch.tensor([s["lens"][b] for b in seqs], device="cuda")[:, None]
        c = torch.tensor([s["counts"][b] for b in seqs], device="cuda")[:, None]
        i = a + torch.arange(nq, device="cuda")[None]
        own_row = i < c
        p = (n - c + i)  # [s, nq] slots of the queries
        # the columns: the sinks, then every slot from the first query's window to the last query
        width = case["window"] if case["window"] else longest
        lo = (n - c + a - width + 1).clamp(min=0)
        span = min(longest, width + nq - 1)
        if len(seqs) == 1:
            span = min(span, int(s["lens"][seqs[0]] - s["counts"][seqs[0]] + a + nq))
        far = lo + torch.arange(span, device="cuda")[None]
        near = torch.arange(sinks, device="cuda")[None].expand(len(seqs), sinks)
        j = torch.cat([near, far], 1)[:, None]  # [s, 1, cols]
        is_sink = torch.arange(sinks + span, device="cuda") < sinks
        back = p[:, :, None] - j
        live = (back >= 0) & (j < n[:, :, None]) & torch.where(is_sink, j < sinks, (back < width) & (j >= sinks))
        j = j[:, 0].clamp(max=longest - 1)
        b = torch.tensor(seqs, device="cuda")
        at = j + (s["start"][b].long()[:, None] if s["start"] is not None else 0)
        at = torch.minimum(at, torch.full_like(at, s["table"].shape[1] * ps - 1))
        page, off = torch.gather(s["table"][b], 1, at // ps).long(), at % ps
        live = live[:, None].expand(len(seqs), g, nq, sinks + span)
        if case["dead"]:
            pos = s["pos"].view(nb, -1, s["pos"].shape[1])[b]
            alive = torch.gather(pos, 2, j[:, None].expand(-1, pos.shape[1], -1)) >= 0
            live = live & alive[:, :, None]
        row = torch.tensor([s["row0s"][x] for x in seqs], device="cuda")[:, None] + i
        q = q_all[torch.where(own_row, row, torch.zeros_like(row))].float()  # [s, nq, g, G, d]
        k = s["k"][1][page, :, off].float()  # [s, cols, g, d]
        z = torch.matmul(q.permute(0, 2, 3, 1, 4).flatten(2, 3), k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
        z = z.unflatten(2, (h // g, nq))
        w = _plain_softmax(z, live[:, :, None])
        v = s["v"][1][page, :, off].float()
        o = torch.matmul(w.flatten(2, 3), v.transpose(1, 2)).unflatten(2, (h // g, nq))
        o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)  # [s, nq, h, d]
        s["out"][row[own_row]] = o[own_row].to(s["out"].dtype)
    return {"out": s["out"]}


# ---------------------------------------------------------------- in 64 bits
def _rows64(s, b, n, i):
    """K and V of the first n slots of sequence b, KV head i."""
    at = torch.arange(n, device="cuda") + s["starts"][b]
    ps = s["case"]["page"]
    page = s["table"][b].long()[at // ps]
    return s["k"][1][page, i, at % ps].double(), s["v"][1][page, i, at % ps].double()


def exact(case, seed):
    s = _inputs(case, seed)
    h, g, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    nb, per = len(s["lens"]), s["pos"].shape[0] // len(s["lens"])
    grp = h // g
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "prefix":
        score = torch.zeros(s["pos"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["lens"]):
            for i in range(g):
                k, v = _rows64(s, b, n, i)
                r = b * per + (i if per > 1 else 0)
                z = s["q"][b, i * grp:(i + 1) * grp].double() @ k.T / math.sqrt(d)
                if case["dead"]:
                    z[:, s["pos"][r, :n] < 0] = -math.inf
                p = torch.nan_to_num(torch.softmax(z, -1), nan=0.0)  # (a row without a live slot)
                out[b, i * grp:(i + 1) * grp] = p @ v
                score[r, :n] += p.sum(0) / (grp if per > 1 else h)
        return {"out": out, "score": score} if case["score"] else {"out": out}
    if work(case)["flops"] > 4.0e12:
        return None
    for b, n in enumerate(s["lens"]):
        c, r0 = s["counts"][b], s["row0s"][b]
        for i in range(g):
            k, v = _rows64(s, b, n, i)
            r = b * per + (i if per > 1 else 0)
            for a in range(0, c, 2048):
                e = min(c, a + 2048)
                p_lo, p_hi = n - c + a, n - c + e - 1
                # the slots that some query of the block sees
                near = set() if not case["window"] else set(range(min(case["sinks"], p_hi + 1)))
                from_ = max(0, p_lo - case["window"] + 1) if case["window"] else 0
                cols = torch.tensor(sorted(x for x in near if x < from_) + list(range(from_, p_hi + 1)), device="cuda")
                p = torch.arange(p_lo, p_hi + 1, device="cuda")[:, None]
                seen = cols[None] <= p
                if case["window"]:
                    seen &= (cols[None] > p - case["window"]) | (cols[None] < case["sinks"])
                if case["dead"]:
                    seen &= (s["pos"][r, cols] >= 0)[None]
                for x in range(grp):
                    head = i * grp + x
                    z = s["qkv"][r0 + a:r0 + e, head * d:(head + 1) * d].double() @ k[cols].T / math.sqrt(d)
                    z.masked_fill_(~seen, -math.inf)
                    w = torch.nan_to_num(torch.softmax(z, -1), nan=0.0)
                    out[r0 + a:r0 + e, head] = w @ v[cols]
    return {"out": out}
