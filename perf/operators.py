"""The 4-bit cache and the page operators as cases that can be timed and compared.

A case is one of four kinds:
  attend   ikv_q4_attend_score: one layer's decode attention over a paged cache held in 4 bits,
           with or without the score of its tokens;
  store    ikv_q4_store and ikv_q4_load: rows of K and V quantised into the pages, and read back;
  fork     a sampling step over shared pages: ikv_pages_release of the sequences that ended,
           ikv_pages_fork of those that go on into their places, ikv_pages_writable for the next
           token of all of them;
  compact  ikv_pages_compact: the survivors of an eviction gathered into pages of their own, the
           old ones given back.

A row of D channels is held as D / 2 bytes of codes and D / 32 scales, one for each group of 32
channels.  Byte u * (D / 16) + 2 * y + h (u < 8, y < D / 32, h < 2) holds channels
32 y + 4 u + 2 h (low half) and the one after it; a code is a sign and one of eight magnitudes.
The plain forms below compute the same things from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MIDPOINTS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)
TINY, HUGE = 2.0 ** -120, 2.0 ** 127  # groups below read as zeros, above as NaN


def _attend(name, **kw):
    c = {"name": name, "kind": "attend", "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16",
         "page": 64, "len_lo": 3277, "len_hi": 3277, "gran": "seq", "score": True, "dead": 0.0, "start": 0}
    c.update(kw)
    return c


def _store(name, **kw):
    c = {"name": name, "kind": "store", "batch": 1, "layers": 1, "kv_heads": 8, "head_dim": 128, "dtype": "bf16",
         "page": 64, "len_lo": 4096, "len_hi": 4096, "newest": 0}
    c.update(kw)
    return c


def _fork(name, **kw):
    c = {"name": name, "kind": "fork", "parents": 1, "ways": 4, "layers": 32, "kv_heads": 8, "head_dim": 128,
         "dtype": "bf16", "page": 64, "len_lo": 8192, "len_hi": 8192}
    c.update(kw)
    return c


def _compact(name, **kw):
    c = {"name": name, "kind": "compact", "batch": 1, "layers": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16",
         "page": 64, "len_lo": 32768, "len_hi": 32768, "budget": 0.1, "same": 0.0, "start": 0, "gran": "seq"}
    c.update(kw)
    return c


def listed():
    return [
        # single-stream decode of the Llama-3.1-8B shape, a 32k prompt evicted to its 10% budget:
        # one layer of a steady step, where latency counts
        _attend("attend_b1_3k"),
        # the same before the eviction: the whole prompt is attended and scored
        _attend("attend_b1_32k", len_lo=32769, len_hi=32769),
        # batched serving with ragged lengths, small pages, evicted tokens still in place as
        # dead slots, sequences that start inside a page
        _attend("attend_b16_ragged", batch=16, page=16, len_lo=4096, len_hi=8192, dead=0.02, start=21),
        # the largest: Qwen-2.5-7B shape (group of 7) at 16k, a step between two refreshes
        # (no scores), a utility row for each KV head
        _attend("attend_qwen_b32_16k", batch=32, q_heads=28, kv_heads=4, page=128, len_lo=12000, len_hi=16384,
                gran="kvhead", score=False),
        # 32-bit queries and outputs (accuracy studies), heads of 64
        _attend("attend_f32_d64", batch=8, q_heads=16, kv_heads=4, head_dim=64, dtype="f32", page=16, len_lo=2000,
                len_hi=4096),
        # the newest token of a batch in every layer: launches and latency only
        _store("store_newest_b32", batch=32, layers=28, kv_heads=4, len_lo=4096, len_hi=16384, newest=1),
        # a 32k prompt, four layers of it at a time, out of the projection's K | V rows
        _store("store_prompt_32k", layers=4, len_lo=32768, len_hi=32768),
        # ragged short prompts packed one behind another, 32-bit rows, heads of 64
        _store("store_ragged_f32", batch=24, layers=2, kv_heads=2, head_dim=64, dtype="f32", page=16, len_lo=17,
               len_hi=1021),
        # a tiny cache: four samples of one short prompt
        _fork("fork_tiny_f32", ways=3, layers=2, kv_heads=2, head_dim=64, dtype="f32", len_lo=513, len_hi=513),
        # sixteen samples of each of two 8k prompts, 32 layers
        _fork("fork_2x16", parents=2, ways=15, len_lo=8100, len_hi=8192),
        # the first eviction of a 32k prompt: a tenth stays, its pages come back
        _compact("compact_first_b1_32k"),
        # a batch held in 4 bits whose shared prompts are left alone: the tail of each sequence is
        # evicted, then read back
        _compact("compact_q4_b16", batch=16, layers=8, dtype="q4", page=16, len_lo=2048, len_hi=4096, budget=0.75,
                 same=0.5),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_LIMIT = {"attend": 2.6e8, "store": 1.3e9, "fork": 3.7e8, "compact": 8.0e8}  # bytes of a drawn pass


def draw(rng):
    while True:
        c = _draw(rng)
        if work(c)["bytes"] <= _LIMIT[c["kind"]] and _held(c) <= 6.0e9:
            return c


def _held(c):
    """Bytes of a drawn case's inputs, roughly."""
    per = c["kv_heads"] * c["head_dim"] * 8 * c.get("layers", 1)
    return per * c["len_hi"] * (c.get("batch") or c["parents"] * (1 + c["ways"]))


def _draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "store", "fork", "compact"])
    hi = _logint(rng, 1, 40000)
    lens = {"len_lo": max(1, int(hi * rng.choice([0.1, 0.5, 1.0]))), "len_hi": hi}
    shape = {"kv_heads": rng.choice([1, 2, 4, 8]), "head_dim": rng.choice([128, 128, 64]),
             "dtype": rng.choice(["bf16", "bf16", "f32"]), "page": rng.choice([16, 48, 64, 128])}
    if kind == "attend":
        c = _attend("", batch=_logint(rng, 1, 48), gran=rng.choice(["seq", "kvhead"]), score=rng.random() < 0.6,
                    dead=rng.choice([0.0, 0.0, 0.03, 0.5]), start=rng.choice([0, 0, 5, 77]), **lens, **shape)
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 4, 7, 8])
    elif kind == "store":
        c = _store("", batch=_logint(rng, 1, 48), layers=rng.choice([1, 2, 4, 28, 32]), newest=rng.choice([0, 0, 1]),
                   **lens, **shape)
    elif kind == "fork":
        c = _fork("", parents=rng.choice([1, 1, 2, 4]), ways=_logint(rng, 1, 24), layers=rng.choice([2, 8, 28, 32]),
                  **lens, **shape)
    else:
        c = _compact("", batch=_logint(rng, 1, 24), layers=rng.choice([2, 8, 28, 32]),
                     budget=rng.choice([0.1, 0.25, 0.5, 0.9]), same=rng.choice([0.0, 0.0, 0.5, 0.9]),
                     start=rng.choice([0, 0, 37]), gran=rng.choice(["seq", "seq", "kvhead"]), **lens, **shape)
        if rng.random() < 0.5:
            c["dtype"] = "q4"
    del c["name"]
    return c


# ---------------------------------------------------------------- sizes
def _spread(lo, hi, n):
    """n lengths over [lo, hi], ragged and fixed by the sizes alone."""
    if lo == hi or n == 1:
        return [hi] * n
    return [lo + (hi - lo) * ((i * 7919 + 3) % 997) // 996 for i in range(n)]


def _row_bytes(case):
    """Bytes of a cached row of K (or V)."""
    d = case["head_dim"]
    return {"bf16": 2 * d, "f32": 4 * d, "q4": d // 2 + d // 16}[case["dtype"]]


def _lens(case):
    return _spread(case["len_lo"], case["len_hi"], case["parents"] if case["kind"] == "fork" else case["batch"])


def _budgets(case):
    return [max(1, int(n * case["budget"])) for n in _lens(case)]


def work(case):
    lens, d, g = _lens(case), case["head_dim"], case["kv_heads"]
    eb = 4 if case["dtype"] == "f32" else 2
    q4 = d // 2 + d // 16
    if case["kind"] == "attend":
        tok, h = sum(lens), case["q_heads"]
        by = tok * g * 2 * q4 + 2 * case["batch"] * h * d * eb
        if case["score"]:
            by += 4 * tok * (g if case["gran"] == "kvhead" else 1)
        return {"bytes": by, "flops": 4 * tok * h * d}
    if case["kind"] == "store":
        rows = (len(lens) if case["newest"] else sum(lens)) * g * 2 * case["layers"]
        return {"bytes": rows * 2 * (d * eb + q4), "flops": 4 * rows * d}
    row = _row_bytes(case) * g * 2 * case["layers"]
    if case["kind"] == "fork":
        n = case["parents"] * case["ways"]
        moved = sum(case["ways"] * (x % case["page"]) for x in lens)
        return {"bytes": 2 * moved * row + n * (case["len_hi"] // case["page"] + 1) * 8, "flops": 0}
    moved, back = 0, 0
    for n, b in zip(lens, _budgets(case)):
        moved += b - min(b, int(case["same"] * b))
        back += b
    by = 2 * moved * row
    if case["dtype"] == "q4":
        by += back * (row + 2 * d * g * 2 * case["layers"])
    return {"bytes": by, "flops": 0}


# ---------------------------------------------------------------- 4 bits, plainly
def _plain_scale(x):
    """[..., D] fp32 -> [..., D / 32] bf16: the smallest s with 6 s >= the group's largest magnitude."""
    a = x.unflatten(-1, (-1, 32)).abs().amax(-1)
    low = ((a * (1.0 / 6.0)).view(torch.int32) & -65536).view(torch.float32)
    up = (low.view(torch.int32) + 65536).view(torch.float32)
    s = torch.where(low * 6.0 < a, up, low)
    s = torch.where(a < TINY, torch.zeros_like(s), s)
    s = torch.where(a <= HUGE, s, torch.full_like(s, math.nan))
    return s.to(torch.bfloat16)


def _plain_quantise(x):
    """[..., D] -> codes [..., D / 2] uint8 and scales [..., D / 32] bf16."""
    x = x.float()
    s = _plain_scale(x)
    y = x.unflatten(-1, (-1, 32))
    w = s.float().unsqueeze(-1)
    mag = sum(((y.abs() >= m * w) & (w > 0)).to(torch.uint8) for m in MIDPOINTS)
    code = (mag | ((y < 0).to(torch.uint8) << 3)).unflatten(-1, (8, 2, 2))  # [..., y, u, h, pair]
    both = code[..., 0] | (code[..., 1] << 4)
    return both.transpose(-3, -2).flatten(-3), s  # [..., u, y, h]


def _plain_values(codes, s):
    """The fp32 values that codes [..., D / 2] and scales [..., D / 32] stand for."""
    n = codes.shape[-1] // 16
    both = codes.unflatten(-1, (8, n, 2)).transpose(-3, -2)  # [..., y, u, h]
    code = torch.stack([both & 15, both >> 4], -1).flatten(-3)  # [..., y, 32]
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    return (table[code.long()] * s.float().unsqueeze(-1)).flatten(-2)


# ---------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _normal(shape, gen, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def prepare(case, seed):
    s = {"attend": _inputs_attend, "store": _inputs_store, "fork": _inputs_fork,
         "compact": _inputs_compact}[case["kind"]](case, seed)
    s["case"] = case
    if own:  # the descriptors and the workspace that a program keeps
        s["plan"] = {"attend": _plan_attend, "store": _plan_store, "fork": _plan_pages,
                     "compact": _plan_pages}[case["kind"]](s)
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attend": _own_attend, "store": _own_store, "fork": _own_fork, "compact": _own_compact}[kind](state)
    return {"attend": _plain_attend, "store": _plain_store, "fork": _plain_fork,
            "compact": _plain_compact}[kind](state)


def _shape(case, batch, layers, q_heads, dtype=None):
    from paper_2609_03515_gb300 import ikv

    return ikv.ikv_shape(batch, layers, q_heads, case["kv_heads"], case["head_dim"],
                         ikv.IKV_F32 if (dtype or case["dtype"]) == "f32" else ikv.IKV_BF16,
                         ikv.IKV_GRAN_KVHEAD if case.get("gran") == "kvhead" else ikv.IKV_GRAN_SEQ)


def _cache(s, k, v, table, lens, max_len, dead=False):
    from paper_2609_03515_gb300 import ikv

    ptr = lambda name: s[name].data_ptr() if s.get(name) is not None else None  # noqa: E731
    return ikv.ikv_cache(k.data_ptr(), v.data_ptr(), table.data_ptr(), k.shape[1], s["case"]["page"], table.shape[1],
                         lens.data_ptr(), ptr("pos"), ptr("next_pos"), max_len, ptr("start"), 1 if dead else 0, None, 0)


# ---------------------------------------------------------------- attend
def _inputs_attend(case, seed):
    gen = _generator(seed)
    nb, g, d, ps = case["batch"], case["kv_heads"], case["head_dim"], case["page"]
    lens = _lens(case)
    starts = [(case["start"] * (b + 1)) % 211 if case["start"] else 0 for b in range(nb)]
    max_pages = max((x + n + ps - 1) // ps for x, n in zip(starts, lens)) + 1
    cap = max_pages * ps
    table = torch.randperm(nb * max_pages, generator=gen, device="cuda").to(torch.int32).view(nb, max_pages)
    s = {"table": table, "len": _i32(lens), "start": _i32(starts) if case["start"] else None}
    # two layers: the second is attended.  Keys around a direction of their head for one token
    # in a hundred, the first four tokens scaled (attention sinks), the rest normal
    u = torch.nn.functional.normalize(_normal((g, d), gen), dim=-1) * 8.0
    heavy = torch.rand(nb * max_pages, ps, generator=gen, device="cuda") < 0.01
    for name in ("k", "v"):
        codes, scales = [], []
        for layer in range(2):
            x = _normal((nb * max_pages, g, ps, d), gen)
            if name == "k":
                x = torch.where(heavy[:, None, :, None], 3.0 * u[None, :, None] + 0.3 * x, x)
                sink = torch.zeros(nb, cap, dtype=torch.bool, device="cuda")
                slot = torch.arange(cap, device="cuda")
                first = _i32(starts)[:, None]
                sink |= (slot >= first) & (slot < first + 4)
                page_sink = torch.zeros(nb * max_pages, ps, dtype=torch.bool, device="cuda")
                page_sink[table.long()] = sink.view(nb, max_pages, ps)
                x = torch.where(page_sink[:, None, :, None], 4.0 * x, x)
            c, z = _plain_quantise(x)
            codes.append(c)
            scales.append(z)
        s[name], s[name + "s"] = torch.stack(codes), torch.stack(scales)
    w = u.repeat_interleave(case["q_heads"] // g, 0)[None] + 0.5 * _normal((nb, case["q_heads"], d), gen)
    s["q"] = (8.0 * torch.nn.functional.normalize(w, dim=-1)).to(DTYPES[case["dtype"]])
    rows = nb * g if case["gran"] == "kvhead" else nb
    s["pos"] = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(rows, 1)
    if case["dead"]:
        s["pos"][torch.rand(rows, cap, generator=gen, device="cuda") < case["dead"]] = -1
    s["next_pos"] = s["len"].clone()
    s["out"] = torch.zeros_like(s["q"])
    s["score"] = torch.zeros(rows, cap, device="cuda") if case["score"] else None
    return s


def _plan_attend(s):
    from paper_2609_03515_gb300 import ikv

    case = s["case"]
    shape = _shape(case, case["batch"], 2, case["q_heads"])
    cache = _cache(s, s["k"], s["v"], s["table"], s["len"], max(_lens(case)), case["dead"] > 0)
    n = ikv.ikv_attend_workspace_size(shape, cache)
    return {"ikv": ikv, "shape": shape, "cache": cache, "q4": ikv.ikv_q4(s["ks"].data_ptr(), s["vs"].data_ptr()),
            "ws": torch.empty(n, dtype=torch.uint8, device="cuda"), "n": n}


def _own_attend(s):
    p = s["plan"]
    p["ikv"].ikv_q4_attend_score(p["shape"], p["cache"], p["q4"], 1, s["q"], s["out"], s["score"], None, 0.0, p["ws"],
                                 p["n"], torch.cuda.current_stream())
    return {"out": s["out"], "score": s["score"]} if s["score"] is not None else {"out": s["out"]}


def _plain_attend(s):
    case = s["case"]
    nb, h, g, d, ps = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    n = max(_lens(case))
    slot = torch.arange(n, device="cuda")[None].expand(nb, n)
    at = slot + s["start"][:, None] if s["start"] is not None else slot
    at = torch.minimum(at, torch.full_like(at, s["table"].shape[1] * ps - 1))
    page, off = torch.gather(s["table"], 1, at // ps).long(), at % ps
    k = _plain_values(s["k"][1][page, :, off], s["ks"][1][page, :, off])  # [b, n, g, d]
    v = _plain_values(s["v"][1][page, :, off], s["vs"][1][page, :, off])
    live = (slot < s["len"][:, None])[:, None].expand(nb, g, n)
    if case["dead"]:
        live = live & (s["pos"].view(nb, -1, s["pos"].shape[1])[:, :, :n] >= 0)
    z = torch.matmul(s["q"].float().view(nb, g, h // g, d), k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    z = torch.where(live[:, :, None], z, torch.full_like(z, -math.inf))
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    sums = e.sum(-1, keepdim=True)
    p = e / torch.where(sums > 0, sums, torch.ones_like(sums))
    v = torch.where(live.transpose(1, 2)[..., None], v, torch.zeros_like(v))
    s["out"].copy_(torch.matmul(p, v.transpose(1, 2)).reshape(nb, h, d))
    if s["score"] is None:
        return {"out": s["out"]}
    rows = s["score"].shape[0]
    pooled = p.mean(2).view(rows, n) if case["gran"] == "kvhead" else p.view(nb, h, n).mean(1)
    inside = slot < s["len"][:, None]
    s["score"][:, :n] = torch.where(inside.repeat_interleave(rows // nb, 0), pooled, s["score"][:, :n])
    return {"out": s["out"], "score": s["score"]}


def _values64(codes, s):
    """Codes [..., D / 2] and scales [..., D / 32] as fp64 [..., D], channel by channel."""
    d = codes.shape[-1] * 2
    ch = torch.arange(d, device=codes.device)
    byte = (ch % 32) // 4 * (d // 16) + 2 * (ch // 32) + (ch % 4) // 2
    c = (codes[..., byte].to(torch.int64) >> (4 * (ch % 2))) & 15
    e, m = (c >> 1) & 3, (c & 1).double()
    mag = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.pow(2.0, e.double() - 1.0))
    return torch.where(c >= 8, -mag, mag) * s[..., ch // 32].double()


def _exact_attend(case, seed):
    s = _inputs_attend(case, seed)
    nb, h, g, d, ps = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    rows = s["pos"].shape[0]
    score = torch.zeros(s["pos"].shape, dtype=torch.float64, device="cuda")
    per = rows // nb
    for b, n in enumerate(_lens(case)):
        at = torch.arange(n, device="cuda") + (int(s["start"][b]) if s["start"] is not None else 0)
        page, off = s["table"][b, at // ps].long(), at % ps
        for i in range(g):
            k = _values64(s["k"][1][page, i, off], s["ks"][1][page, i, off])
            v = _values64(s["v"][1][page, i, off], s["vs"][1][page, i, off])
            r = b * per + (i if per > 1 else 0)
            live = s["pos"][r, :n] >= 0
            z = s["q"][b, i * (h // g):(i + 1) * (h // g)].double() @ k.T / math.sqrt(d)
            z[:, ~live] = -math.inf
            p = torch.softmax(z, -1) if bool(live.any()) else torch.zeros_like(z)
            out[b, i * (h // g):(i + 1) * (h // g)] = p @ v
            score[r, :n] += p.sum(0) / (h // g if per > 1 else h)
    return {"out": out, "score": score} if case["score"] else {"out": out}


# ---------------------------------------------------------------- store
def _inputs_store(case, seed):
    gen = _generator(seed)
    nb, layers, g, d, ps = case["batch"], case["layers"], case["kv_heads"], case["head_dim"], case["page"]
    lens = _lens(case)
    counts = [1] * nb if case["newest"] else lens
    first = [n - 1 for n in lens] if case["newest"] else [0] * nb
    max_pages = (max(lens) + ps - 1) // ps
    pages = nb * max_pages if not case["newest"] else nb + 1  # newest: a token's page each, the others unused
    if case["newest"]:
        table = torch.zeros(nb, max_pages, dtype=torch.int32, device="cuda")
        table.scatter_(1, (_i32(lens)[:, None] - 1).long() // ps, _i32(list(range(1, nb + 1)))[:, None])
    else:
        table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).view(nb, max_pages)
    total = sum(counts)
    kv = _normal((layers, total, 2, g, d), gen).to(DTYPES[case["dtype"]])  # a projection's K | V rows
    kv[:, :, :, :, 5] *= 6.0  # a loud channel
    s = {"table": table, "len": _i32(lens), "kv": kv, "first": _i32(first), "count": _i32(counts),
         "row0": _i32([sum(counts[:b]) for b in range(nb)])}
    for name in ("k", "v"):
        s[name] = torch.zeros(layers, pages, g, ps, d // 2, dtype=torch.uint8, device="cuda")
        s[name + "s"] = torch.zeros(layers, pages, g, ps, d // 32, dtype=torch.bfloat16, device="cuda")
        s[name + "_out"] = torch.zeros(layers, total, g, d, dtype=kv.dtype, device="cuda")
    # sequence, slot, page and offset of every packed row
    seq = torch.repeat_interleave(torch.arange(nb, device="cuda"), s["count"].long())
    slot = torch.arange(total, device="cuda") - s["row0"].long()[seq] + s["first"].long()[seq]
    s["page"], s["off"] = table[seq, slot // ps].long(), slot % ps
    return s


def _plan_store(s):
    from paper_2609_03515_gb300 import ikv

    case, kv = s["case"], s["kv"]
    g, d, total = case["kv_heads"], case["head_dim"], kv.shape[1]
    r0 = s["row0"].data_ptr()
    return {"ikv": ikv, "shape": _shape(case, case["batch"], case["layers"], g),
            "cache": _cache(s, s["k"], s["v"], s["table"], s["len"], max(_lens(case))),
            "q4": ikv.ikv_q4(s["ks"].data_ptr(), s["vs"].data_ptr()),
            "src": ikv.ikv_rows(total * 2 * g * d, 0, 2 * g * d, d, r0),
            "dst": ikv.ikv_rows(total * g * d, 0, g * d, d, r0), "most": 1 if case["newest"] else max(_lens(case))}


def _own_store(s):
    p, kv, layers = s["plan"], s["kv"], s["case"]["layers"]
    st = torch.cuda.current_stream()
    p["ikv"].ikv_q4_store(p["shape"], p["cache"], p["q4"], 0, layers, kv[:, :, 0], kv[:, :, 1], p["src"], s["first"],
                          s["count"], p["most"], st)
    p["ikv"].ikv_q4_load(p["shape"], p["cache"], p["q4"], 0, layers, s["k_out"], s["v_out"], p["dst"], s["first"],
                         s["count"], p["most"], st)
    return {"k": s["k_out"], "v": s["v_out"], "ks": s["ks"], "vs": s["vs"]}


def _plain_store(s):
    page, off = s["page"], s["off"]
    for i, name in enumerate(("k", "v")):
        c, z = _plain_quantise(s["kv"][:, :, i])
        s[name][:, page, :, off] = c.transpose(0, 1)
        s[name + "s"][:, page, :, off] = z.transpose(0, 1)
        back = _plain_values(s[name][:, page, :, off], s[name + "s"][:, page, :, off])
        s[name + "_out"].copy_(back.transpose(0, 1))
    return {"k": s["k_out"], "v": s["v_out"], "ks": s["ks"], "vs": s["vs"]}


def _exact_store(case, seed):
    s = _inputs_store(case, seed)
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    got = {}
    for i, name in enumerate(("k", "v")):
        got[name] = torch.zeros(s[name + "_out"].shape, dtype=torch.float64, device="cuda")
        got[name + "s"] = torch.zeros(s[name + "s"].shape, dtype=torch.float64, device="cuda")
        for layer in range(case["layers"]):
            x = s["kv"][layer, :, i].double()
            x = x.view(*x.shape[:-1], -1, 32)
            a = x.abs().amax(-1)
            t = a / torch.full_like(a, 6.0)  # (a tensor: by a number it would be a product with its inverse)
            # the step of bf16 at t, as a power of two put together from its exponent
            ulp = ((torch.frexp(t).exponent.to(torch.int64) - 8 + 1023) << 52).view(torch.float64)
            z = torch.ceil(t / ulp) * ulp
            r = x.abs() / z[..., None]
            # the nearest magnitude, the larger of two as near
            up = torch.bucketize(r, grid, right=True).clamp(max=7)
            lo = grid[up - 1]
            mag = torch.where(r - lo >= grid[up] - r, grid[up], lo)
            got[name][layer] = (torch.sign(x) * mag * z[..., None]).flatten(-2)
            got[name + "s"][layer, s["page"], :, s["off"]] = z
    return {"k": got["k"], "v": got["v"], "ks": got["ks"], "vs": got["vs"]}


# ---------------------------------------------------------------- pages
def _planes(case, pages, gen):
    """The paged arrays of a cache, K's and V's alike: [layers][pages][kv_heads][page][row]."""
    at = (case["layers"], pages, case["kv_heads"], case["page"])
    d = case["head_dim"]
    if case["dtype"] != "q4":
        return [_normal(at + (d,), gen, DTYPES[case["dtype"]]) for _ in range(2)]
    made = [torch.randint(0, 256, at + (d // 2,), dtype=torch.uint8, generator=gen, device="cuda") for _ in range(2)]
    return made + [_normal(at + (d // 32,), gen).abs().to(torch.bfloat16) for _ in range(2)]


def _books(s, **tensors):
    """The small tensors that a pass rewrites, as views of one buffer that one copy rewinds."""
    sizes = [(t.numel() + 3) // 4 * 4 for t in tensors.values()]
    s["books"] = torch.zeros(sum(sizes), dtype=torch.int32, device="cuda")
    at = 0
    for (name, t), n in zip(tensors.items(), sizes):
        s[name] = s["books"][at:at + t.numel()].view(t.dtype).view(t.shape)
        s[name].copy_(t)
        at += n
    s["saved"] = s["books"].clone()


def _utility(shape, gen):
    return torch.exp(3.0 * _normal(shape, gen) - 9.0)


def _inputs_fork(case, seed):
    gen = _generator(seed)
    ps, parents, ways = case["page"], case["parents"], case["ways"]
    nb, lens = parents * (1 + ways), _lens(case)
    max_pages = (max(lens) + ps - 1) // ps + 2
    held = [(n + ps - 1) // ps for n in lens]
    ended = 3  # pages that a sequence which ended still holds
    n_pages = 1 + sum(held) + (nb - parents) * min(ended, max_pages)
    ids = 1 + torch.randperm(n_pages - 1, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(nb, max_pages, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(nb):
        n = held[b] if b < parents else min(ended, max_pages)
        table[b, :n] = ids[at:at + n]
        at += n
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    cap = max_pages * ps
    s = {"planes": _planes(case, n_pages, gen),
         "src": _i32([b for b in range(parents) for _ in range(ways)]), "dst": _i32(list(range(parents, nb)))}
    lens = _i32(lens + [0] * (nb - parents))
    pos = torch.full((nb, cap), -1, dtype=torch.int32, device="cuda")
    pos[:parents] = torch.arange(cap, dtype=torch.int32, device="cuda")
    ema = torch.zeros(nb, cap, device="cuda")
    ema[:parents] = _utility((parents, cap), gen)
    _books(s, table=table, refs=refs, len=lens, next_pos=lens, pos=pos, ema=ema.view(torch.int32))
    s["ema"] = s["ema"].view(torch.float32)
    s["max_len"] = case["len_hi"]
    return s


def _inputs_compact(case, seed):
    gen = _generator(seed)
    ps, nb, g = case["page"], case["batch"], case["kv_heads"]
    lens, budgets = _lens(case), _budgets(case)
    starts = [case["start"] * b % 97 if case["start"] else 0 for b in range(nb)]
    max_pages = max((x + n + ps - 1) // ps for x, n in zip(starts, lens)) + 1
    cap = max_pages * ps
    per = g if case["gran"] == "kvhead" else 1
    # the pages of every sequence, and room for the survivors
    held = [(x + n + ps - 1) // ps for x, n in zip(starts, lens)]
    n_pages = 1 + sum(held) + sum((x + b + ps - 1) // ps for x, b in zip(starts, budgets))
    ids = 1 + torch.randperm(n_pages - 1, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(nb, max_pages, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[0] = 1
    keep = torch.zeros(nb * per, cap, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(nb):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
        # the first `same` of the budget stays where it is, the rest is drawn
        f = min(budgets[b], int(case["same"] * budgets[b]))
        for r in range(per):
            rest = f + torch.randperm(lens[b] - f, generator=gen, device="cuda")[:budgets[b] - f]
            row = torch.cat([torch.arange(f, device="cuda"), torch.sort(rest).values])
            keep[b * per + r, :budgets[b]] = row.to(torch.int32)
    refs[table.flatten().long()] = 1
    s = {"planes": _planes(case, n_pages, gen), "keep": keep,
         "keep_len": _i32([x for x in budgets for _ in range(per)]), "start": _i32(starts) if case["start"] else None,
         "max_len": max(lens)}
    n = _i32(lens)
    pos = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(nb * per, 1)
    _books(s, table=table, refs=refs, len=n, next_pos=n, pos=pos, ema=_utility((nb * per, cap), gen).view(torch.int32))
    s["ema"] = s["ema"].view(torch.float32)
    if case["dtype"] == "q4":
        d = case["head_dim"]
        s["first"] = torch.zeros(nb, dtype=torch.int32, device="cuda")
        s["row0"] = _i32([sum(budgets[:b]) for b in range(nb)])
        s["back"] = [torch.zeros(case["layers"], sum(budgets), g, d, dtype=torch.bfloat16, device="cuda")
                     for _ in range(2)]
        seq = torch.repeat_interleave(torch.arange(nb, device="cuda"), _i32(budgets).long())
        s["seq"], s["slot"] = seq, torch.arange(sum(budgets), device="cuda") - s["row0"].long()[seq]
    return s


def _plan_pages(s):
    from paper_2609_03515_gb300 import ikv

    case = s["case"]
    nb = s["table"].shape[0]
    shape = _shape(case, nb, case["layers"], case["kv_heads"])
    cache = _cache(s, s["planes"][0], s["planes"][1], s["table"], s["len"], s["max_len"])
    pages = ikv.ikv_pages_of(s["refs"], s["planes"])
    n = ikv.ikv_pages_workspace_size(shape, cache, pages)
    p = {"ikv": ikv, "shape": shape, "cache": cache, "pages": pages, "n": n,
         "ws": torch.empty(n, dtype=torch.uint8, device="cuda")}
    if case["dtype"] == "q4":
        g, d = case["kv_heads"], case["head_dim"]
        total = s["back"][0].shape[1]
        p["q4"] = ikv.ikv_q4(s["planes"][2].data_ptr(), s["planes"][3].data_ptr())
        p["dst"] = ikv.ikv_rows(total * g * d, 0, g * d, d, s["row0"].data_ptr())
        p["most"] = max(_budgets(case))
    return p


def _pages_out(s):
    got = {"table": s["table"], "refs": s["refs"], "len": s["len"], "pos": s["pos"], "ema": s["ema"]}
    got.update({"k": s["back"][0], "v": s["back"][1]} if "back" in s else
               {"k": s["planes"][0], "v": s["planes"][1]})
    return got


def _own_fork(s):
    p, st = s["plan"], torch.cuda.current_stream()
    s["books"].copy_(s["saved"])
    p["ikv"].ikv_pages_release(p["shape"], p["cache"], p["pages"], 0, st)
    p["ikv"].ikv_pages_fork(p["shape"], p["cache"], p["pages"], s["src"].numel(), s["src"], s["dst"], s["ema"], st)
    p["ikv"].ikv_pages_writable(p["shape"], p["cache"], p["pages"], None, None, 1, None, p["ws"], p["n"], st)
    return _pages_out(s)


def _own_compact(s):
    p, st = s["plan"], torch.cuda.current_stream()
    s["books"].copy_(s["saved"])
    p["ikv"].ikv_pages_compact(p["shape"], p["cache"], p["pages"], s["keep"], s["keep_len"], s["ema"], None, p["ws"],
                               p["n"], st)
    if "back" in s:
        p["ikv"].ikv_q4_load(p["shape"], p["cache"], p["q4"], 0, s["case"]["layers"], s["back"][0], s["back"][1],
                             p["dst"], s["first"], s["len"], p["most"], st)
    return _pages_out(s)


def _free_pages(refs):
    """Page numbers, the free ones first and ascending."""
    return torch.argsort((refs > 0).to(torch.int32), stable=True).to(torch.int32)


def _plain_fork(s):
    s["books"].copy_(s["saved"])
    table, refs, ps = s["table"], s["refs"], s["case"]["page"]
    nb, max_pages = table.shape
    lp = torch.arange(max_pages, device="cuda")[None]
    # release: pages that hold no slot in use
    gone = (table > 0) & (lp * ps >= s["len"][:, None])
    refs.scatter_add_(0, table.flatten().long(), -gone.flatten().to(torch.int32))
    table.masked_fill_(gone, 0)
    # fork
    src, dst = s["src"].long(), s["dst"].long()
    for t in (table, s["pos"], s["ema"]):
        t[dst] = t[src]
    for t in (s["len"], s["next_pos"]):
        t[dst] = t[src]
    refs.scatter_add_(0, table[dst].flatten().long(), (table[dst] > 0).flatten().to(torch.int32))
    # the page of every sequence's next slot: its own, a copy of a shared one, or a new one.  Of
    # the sequences that would write a shared page which nobody else holds, the last keeps it
    row = s["len"].long() // ps
    e = table.gather(1, row[:, None])[:, 0].long()
    b = torch.arange(nb, device="cuda")
    shared = (e > 0) & (refs[e] > 1)
    writers = torch.zeros_like(refs).scatter_add_(0, e, shared.to(torch.int32))
    last = torch.full(refs.shape, -1, device="cuda").scatter_reduce_(0, e, torch.where(shared, b, -1), "amax")
    stays = shared & (writers[e] == refs[e]) & (last[e] == b)
    new = (e == 0) | (shared & ~stays)
    copied = shared & ~stays
    to = torch.where(new, _free_pages(refs)[(torch.cumsum(new, 0) - 1).clamp(min=0)].long(), e)
    table.scatter_(1, row[:, None], to[:, None].to(torch.int32))
    refs.scatter_add_(0, e, -copied.to(torch.int32))
    refs.scatter_add_(0, to, new.to(torch.int32))
    held = torch.arange(ps, device="cuda")[None] < (s["len"].long() % ps)[:, None]  # rows in use
    at, off = torch.nonzero(held & copied[:, None], as_tuple=True)
    for t in s["planes"]:
        t[:, to[at], :, off] = t[:, e[at], :, off]
    return _pages_out(s)


def _plain_compact(s):
    s["books"].copy_(s["saved"])
    case, table, refs = s["case"], s["table"], s["refs"]
    ps, g = case["page"], case["kv_heads"]
    nb, max_pages = table.shape
    per = s["pos"].shape[0] // nb
    cap = max_pages * ps
    slot = torch.arange(cap, device="cuda")
    n = s["keep_len"].long()[::per]
    start = s["start"].long() if s["start"] is not None else torch.zeros(nb, dtype=torch.long, device="cuda")
    keep = torch.where(slot[None] < s["keep_len"][:, None], s["keep"], 0).long()
    still = ((keep == slot[None]) & (slot[None] < s["keep_len"][:, None])).to(torch.int32)
    f = torch.cumprod(still, 1).sum(1).view(nb, per).amin(1).long()
    end = (start + n + ps - 1) // ps
    begin = torch.where(f == n, end, (start + f) // ps)  # the first page that is made anew
    lp = torch.arange(max_pages, device="cuda")[None]
    new = (lp >= begin[:, None]) & (lp < end[:, None])
    gone = (table > 0) & (lp >= begin[:, None])
    rank = (torch.cumsum(new.flatten(), 0) - 1).clamp(min=0)
    old = table.clone()
    to = torch.where(new, _free_pages(refs)[rank].view(nb, max_pages), torch.where(gone, 0, table))
    refs.scatter_add_(0, old.flatten().long(), -gone.flatten().to(torch.int32))
    refs.scatter_add_(0, to.flatten().long(), new.flatten().to(torch.int32))
    table.copy_(to)
    # rows that move: slot j of a new page comes from slot keep[j]
    at = start[:, None] + slot[None]
    page = torch.gather(to, 1, (at // ps).clamp(max=max_pages - 1)).long()
    moves = (slot[None] < n[:, None]) & (at // ps >= begin[:, None])
    b, j = torch.nonzero(moves, as_tuple=True)
    dst, dst_off = page[b, j], at[b, j] % ps
    head = torch.arange(g, device="cuda")[None]
    frm = start[b][:, None] + keep.view(nb, per, cap)[b, :, j]  # [moves, per]
    src, src_off = old[b[:, None], frm // ps].long(), frm % ps
    for t in s["planes"]:
        t[:, dst[:, None], head, dst_off[:, None]] = t[:, src, head, src_off]
    inside = slot[None] < s["keep_len"][:, None]
    for t in (s["pos"], s["ema"]):
        t.copy_(torch.where(inside, torch.gather(t, 1, keep), t))
    s["len"].copy_(n)
    if "back" in s:
        seq, sl = s["seq"], s["slot"] + start[s["seq"]]
        page, off = table[seq, sl // ps].long(), sl % ps
        for i in range(2):
            z = _plain_values(s["planes"][i][:, page, :, off], s["planes"][2 + i][:, page, :, off])
            s["back"][i].copy_(z.transpose(0, 1))
    return _pages_out(s)


def _exact_fork(case, seed):
    s = _inputs_fork(case, seed)
    ps, parents = case["page"], case["parents"]
    table, refs = s["table"].tolist(), s["refs"].tolist()
    lens, pos, ema = s["len"].tolist(), s["pos"].clone(), s["ema"].clone()
    nb = len(table)
    for b in range(nb):
        for p, e in enumerate(table[b]):
            if e and p * ps >= lens[b]:
                refs[e] -= 1
                table[b][p] = 0
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        table[b], lens[b] = list(table[a]), lens[a]
        pos[b], ema[b] = pos[a], ema[a]
        for e in table[b]:
            refs[e] += 1 if e else 0
    held = list(refs)
    free = [i for i, r in enumerate(held) if r == 0]
    for b in range(nb):
        p = lens[b] // ps
        e = table[b][p]
        if e and held[e] > 1:
            same = [x for x in range(nb) if lens[x] // ps < len(table[x]) and table[x][lens[x] // ps] == e]
            # (those before b have their copies already)
            if b == max(same) and refs[e] == 1:
                continue
            to = free.pop(0)
            for t in s["planes"]:
                t[:, to, :, :lens[b] % ps] = t[:, e, :, :lens[b] % ps]
            refs[e] -= 1
        elif e == 0:
            to = free.pop(0)
        else:
            continue
        refs[to] = 1
        table[b][p] = to
    return {"table": None, "refs": None, "len": None, "pos": None, "ema": ema.double(), "k": s["planes"][0],
            "v": s["planes"][1]}


def _exact_compact(case, seed):
    s = _inputs_compact(case, seed)
    ps, g, lens, budgets = case["page"], case["kv_heads"], _lens(case), _budgets(case)
    nb, per = len(lens), s["pos"].shape[0] // len(lens)
    ema = s["ema"].clone()
    for r in range(nb * per):
        n = budgets[r // per]
        ema[r, :n] = s["ema"][r, s["keep"][r, :n].long()]
    got = {"table": None, "refs": None, "len": None, "pos": None, "ema": ema.double()}
    if case["dtype"] == "q4":
        for i, name in enumerate(("k", "v")):
            got[name] = torch.zeros(s["back"][i].shape, dtype=torch.float64, device="cuda")
            at = 0
            for b, n in enumerate(budgets):
                for h in range(g):
                    frm = s["keep"][b * per + (h if per > 1 else 0), :n].long()
                    frm = frm + (int(s["start"][b]) if s["start"] is not None else 0)
                    page, off = s["table"][b, frm // ps].long(), frm % ps
                    got[name][:, at:at + n, h] = _values64(s["planes"][i][:, page, h, off],
                                                           s["planes"][2 + i][:, page, h, off])
                at += n
        return got
    table, free = s["table"].tolist(), [i for i, r in enumerate(s["refs"].tolist()) if r == 0]
    planes = [t.clone() for t in s["planes"]]
    for b, n in enumerate(budgets):
        x = int(s["start"][b]) if s["start"] is not None else 0
        rows = [s["keep"][b * per + r, :n].tolist() for r in range(per)]
        f = min(next((j for j in range(n) if row[j] != j), n) for row in rows)
        if f == n:
            continue
        for p in range((x + f) // ps, (x + n + ps - 1) // ps):
            to = free.pop(0)
            j = torch.arange(max(0, p * ps - x), min(n, (p + 1) * ps - x), device="cuda")
            for h in range(g):
                frm = s["keep"][b * per + (h if per > 1 else 0)][j].long() + x
                page = s["table"][b][frm // ps].long()
                for t, old in zip(planes, s["planes"]):
                    t[:, to, h, (j + x) % ps] = old[:, page, h, frm % ps]
    del table
    got.update({"k": planes[0], "v": planes[1]})
    return got


def exact(case, seed):
    return {"attend": _exact_attend, "store": _exact_store, "fork": _exact_fork,
            "compact": _exact_compact}[case["kind"]](case, seed)
