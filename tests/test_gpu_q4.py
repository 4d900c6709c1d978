"""Caches held in 4 bits: store, load, append and decode attention against plain fp64.

Store and load are defined bit for bit, so they are compared exactly.  The bounds of the
attention follow from its roundings:
  weights p * scale are rounded to fp16 (one term for bf16 outputs: 2^-11 of each; two for fp32:
  2^-22), or, below fp16's normal range, to 2^-25 with the largest scale seen at 2^4 or above
  and the largest weight's p at 1 or above;
  queries enter as one fp16 term, exact for bf16, or two (2^-22);
  every sum is fp32, in all an error of some 2^-20 of the sum of its terms' magnitudes, and an
  error d of a logit is a factor 1 + d of its probability;
  bf16 outputs are rounded once more (2^-8 covers it)."""
import math

import pytest
import torch

from paper_2609_03515_gb300 import Q4Cache, ikv

pytestmark = pytest.mark.gpu

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
TORCH = {ikv.IKV_F32: torch.float32, ikv.IKV_BF16: torch.bfloat16}


def quantise(x):
    """The definition, in fp64: codes by channel [..., D] (int64) and scales [..., D / 32]."""
    x = x.double().unflatten(-1, (-1, 32))
    a = x.abs().amax(-1)
    six = torch.full_like(a, 6.0)  # (by a tensor: by a number it would be a product with 1 / 6)
    t = torch.where((a >= 2.0 ** -120) & (a <= 2.0 ** 127), a, torch.ones_like(a)) / six
    ulp = ((torch.frexp(t).exponent.to(torch.int64) - 8 + 1023) << 52).view(torch.float64)
    s = torch.ceil(t / ulp) * ulp
    s = torch.where(a < 2.0 ** -120, torch.zeros_like(s), s)
    s = torch.where(a <= 2.0 ** 127, s, torch.full_like(s, math.nan))
    r = torch.where(s[..., None] > 0, x.abs() / s[..., None], torch.zeros_like(x))
    mag = torch.zeros_like(x, dtype=torch.int64)
    for lo, hi in zip(GRID[:-1], GRID[1:]):
        mag += (r >= (lo + hi) / 2).to(torch.int64)  # nearest, the larger of two as near
    return (mag + 8 * (x < 0)).flatten(-2), s


def values(codes, s):
    table = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64, device=codes.device)
    return table[codes] * s.repeat_interleave(32, -1)


def unpack(raw):
    """Bytes [..., D / 2] -> codes by channel [..., D]."""
    d = raw.shape[-1] * 2
    ch = torch.arange(d, device=raw.device)
    byte = (ch % 32) // 4 * (d // 16) + 2 * (ch // 32) + (ch % 4) // 2
    return (raw[..., byte].to(torch.int64) >> (4 * (ch % 2))) & 15


def same_codes(a, b, s):
    """Equal codes, either sign of zero, anything where the scale is NaN."""
    z = (a & 7 == 0) & (b & 7 == 0)
    return bool((z | (a == b) | s.repeat_interleave(32, -1).isnan()).all())


def noise(c, gen):
    """Anything at all in the pools, NaN scales among it."""
    for t in (c.k, c.v):
        t.random_(0, 256, generator=gen)
    for t in (c.k_scale, c.v_scale):
        t.fill_(math.nan)


def paged(c, pool, b, layer, n, first=0):
    """Rows first .. first + n - 1 of sequence b: [n][kv_heads][row]."""
    at = torch.arange(first, first + n, device="cuda") + int(c.start[b])
    return pool[layer, c.block_table[b, at // c.page_size].long(), :, at % c.page_size]


def make(lens, kvh, G, d, ps, dtype, starts=None, layers=2, gran=ikv.IKV_GRAN_SEQ, room=40):
    c = Q4Cache(len(lens), layers, G * kvh, kvh, d, max(lens) + room, dtype=dtype, page_size=ps, granularity=gran,
                page_perm_seed=3)
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    if starts:
        c.start.copy_(torch.tensor(starts, dtype=torch.int32))
    c.pos.copy_(torch.arange(c.cap, dtype=torch.int32, device="cuda").expand(c.rows, c.cap))
    return c


def hard_rows(shape, gen, dt):
    """Rows with ties, zeros, tiny and huge groups, infinities and NaN among normal ones."""
    x = torch.randn(shape, generator=gen, device="cuda")
    y = x.view(-1, 32)
    n = y.shape[0]
    kind = torch.randint(0, 12, (n,), generator=gen, device="cuda")
    grid = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6], device="cuda")
    ties = grid[torch.randint(0, 15, (n, 32), generator=gen, device="cuda")]
    ties[:, 0] = 6.0  # the scale is then the power of two itself
    ties = ties * torch.exp2(torch.randint(-20, 20, (n, 1), generator=gen, device="cuda").float())
    ties = ties * (1 - 2 * torch.randint(0, 2, (n, 32), generator=gen, device="cuda"))
    y[kind == 0] = ties[kind == 0]
    y[kind == 1] = 0.0
    y[kind == 2] *= 2.0 ** -125
    y[kind == 3] *= 2.0 ** 120
    y[kind == 4] *= 2.0 ** -118
    y[(kind == 5).nonzero()[:, 0], 7] = math.inf
    y[(kind == 6).nonzero()[:, 0], 31] = math.nan
    y[kind == 7] = (ties[kind == 7].double() * (1 + 2.0 ** -23)).float()  # an ulp beside the ties
    y[kind == 8] = (ties[kind == 8].double() * (1 - 2.0 ** -24)).float()
    y[kind == 9, 5:] = 0.0
    y[(kind == 10).nonzero()[:, 0], 3] = 2.0 ** 127 * 1.5
    return x.to(dt)


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
@pytest.mark.parametrize("d,kvh,ps", [(64, 1, 16), (64, 3, 48), (128, 2, 64), (128, 8, 16), (128, 5, 112)])
def test_store_and_load_are_exact(dtype, d, kvh, ps):
    gen = torch.Generator(device="cuda").manual_seed(d + kvh)
    lens = [0, 1, 15, 16, 17, 130, 777]
    firsts = [0, 0, 3, 16, 5, 100, 1]
    c = make([f + n for f, n in zip(firsts, lens)], kvh, 1, d, ps, dtype, starts=[(5 * i) % 23 for i in range(7)],
             layers=3)
    noise(c, gen)
    before = [t.clone() for t in c.planes()]
    total = sum(lens)
    # packed rows, K and V interleaved, a gap between tokens; layers 1 and 2
    kv = hard_rows((2, total, 2, kvh, d + 32), gen, TORCH[dtype])
    k, v = kv[:, :, 0, :, :d], kv[:, :, 1, :, 32:]
    row0 = torch.tensor([sum(lens[:i]) for i in range(7)], dtype=torch.int32, device="cuda")
    first = torch.tensor(firsts, dtype=torch.int32, device="cuda")
    count = torch.tensor(lens, dtype=torch.int32, device="cuda")
    shape, cache, q4 = c.shape(), c.cache(int(c.len.max())), c.q4()
    rows = c.dense_rows(k, row0)
    ikv.ikv_q4_store(shape, cache, q4, 1, 2, k, v, rows, first, count, max(lens))
    back = [torch.full((2, total, kvh, d), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    ikv.ikv_q4_load(shape, cache, q4, 1, 2, back[0], back[1], c.dense_rows(back[0], row0), first, count, max(lens))
    assert ikv.ikv_device_status() == 0
    touched = [torch.zeros(t.shape, dtype=torch.bool, device="cuda") for t in c.planes()]
    for i, (x, codes, scale) in enumerate(((k, c.k, c.k_scale), (v, c.v, c.v_scale))):
        for b, (f, n) in enumerate(zip(firsts, lens)):
            at = torch.arange(f, f + n, device="cuda") + int(c.start[b])
            page, off = c.block_table[b, at // ps].long(), at % ps
            for layer in (1, 2):
                want, s = quantise(x[layer - 1, int(row0[b]):int(row0[b]) + n])
                got = scale[layer, page, :, off].double()
                assert torch.equal(got.nan_to_num(nan=-1.0), s.nan_to_num(nan=-1.0))
                assert same_codes(unpack(codes[layer, page, :, off]), want, s)
                val = values(want, s).to(torch.float32).to(TORCH[dtype])
                assert torch.equal(val.nan_to_num(nan=-1.0),
                                   back[i][layer - 1, int(row0[b]):int(row0[b]) + n].nan_to_num(nan=-1.0))
                touched[i][layer, page, :, off] = True
                touched[2 + i][layer, page, :, off] = True
    for t, was, mark in zip(c.planes(), before, touched):
        assert torch.equal(t[~mark].view(torch.uint8), was[~mark].view(torch.uint8))


def test_store_defaults_and_rows_left_out():
    """first NULL: the newest slots; first < 0: nothing; rows past the slot space: nothing, and the error bit."""
    c = make([5, 0, 40, 64], 2, 2, 64, 16, ikv.IKV_BF16, room=0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(2, 4, 3, 2, 64, generator=gen, device="cuda").to(torch.bfloat16)
    ikv.ikv_q4_store(c.shape(), c.cache(64), c.q4(), 0, 2, x, x, c.dense_rows(x), None, None, 3)
    back, other = torch.zeros_like(x), torch.zeros_like(x)
    ikv.ikv_q4_load(c.shape(), c.cache(64), c.q4(), 0, 2, back, other, c.dense_rows(back), None, None, 3)
    want = values(*quantise(x)).to(torch.bfloat16)
    want[:, 1] = 0
    assert torch.equal(back, want) and torch.equal(other, want)
    held = [t.clone() for t in c.planes()]
    first = torch.tensor([-1, 62, 64, -7], dtype=torch.int32, device="cuda")
    assert ikv.ikv_device_status() == 0
    ikv.ikv_q4_store(c.shape(), c.cache(64), c.q4(), 0, 2, 2 * x, x, c.dense_rows(x), first, None, 3)
    assert ikv.ikv_device_status() == 32
    assert all(torch.equal(a, b) for a, b in zip(held, c.planes()))
    first = torch.tensor([0, 61, 0, 0], dtype=torch.int32, device="cuda")
    count = torch.tensor([0, 3, -4, 100], dtype=torch.int32, device="cuda")  # 100 is cut to 3
    ikv.ikv_q4_store(c.shape(), c.cache(64), c.q4(), 0, 2, x, x, c.dense_rows(x), first, count, 3)
    assert ikv.ikv_device_status() == 0
    for b, f in ((1, 61), (3, 0)):
        got = values(unpack(paged(c, c.k, b, 1, 3, f)), paged(c, c.k_scale, b, 1, 3, f).double())
        assert torch.equal(got, values(*quantise(x[1, b])))


def reference(c, q, layer, b, g, L, live):
    """fp64 output [G][D] and probabilities [G][L], and the sizes that the bounds speak of."""
    G, D = c.q_heads // c.kv_heads, c.head_dim
    K = values(unpack(paged(c, c.k, b, layer, L))[:, g], paged(c, c.k_scale, b, layer, L)[:, g].double())
    V = values(unpack(paged(c, c.v, b, layer, L))[:, g], paged(c, c.v_scale, b, layer, L)[:, g].double())
    K, V = torch.where(live[:, None], K, 0.0), torch.where(live[:, None], V, 0.0)
    x = q[b, g * G:(g + 1) * G].double()
    z = x @ K.T / math.sqrt(D)
    z[:, ~live] = -math.inf
    p = torch.softmax(z, -1) if bool(live.any()) else torch.zeros_like(z)
    zmag = (x.abs() @ K.abs().T / math.sqrt(D)).amax() if L else 0.0
    vs = torch.where(live[:, None], paged(c, c.v_scale, b, layer, L)[:, g].double(), 0.0).amax() if L else 0.0
    return p @ V, p, p @ V.abs(), float(zmag), float(vs)


def check(c, layer, q, out, score, dead, live_rows):
    two = c.dtype == ikv.IKV_F32
    G = c.q_heads // c.kv_heads
    lens = c.len.tolist()
    for b, L in enumerate(lens):
        per = c.rows // len(lens)
        pooled = torch.zeros(per, L, dtype=torch.float64, device="cuda")
        zmax = 0.0
        for g in range(c.kv_heads):
            r = b * per + (g if per > 1 else 0)
            live = live_rows[r, :L]
            o, p, mag, zmag, vs = reference(c, q, layer, b, g, L, live)
            zmax = max(zmax, zmag)
            pooled[g if per > 1 else 0] += p.sum(0) / (G if per > 1 else c.q_heads)
            factor = (2.0 ** -21 if two else 2.0 ** -10) + zmag * 2.0 ** -18 + 2.0 ** -18
            bound = mag * factor + L * 2.0 ** (-36 if two else -25) * 6.0 * vs / 16 + 1e-40
            if not two:
                bound = bound + o.abs() * 2.0 ** -8
            err = (out[b, g * G:(g + 1) * G].double() - o).abs()
            assert bool((err <= bound).all()), (b, L, g, float((err / bound).max()))
        if score is not None and L:
            got = score[b * per:(b + 1) * per, :L].double()
            bound = pooled * (zmax * 2.0 ** -18 + 2.0 ** -18) + 1e-30
            assert bool(((got - pooled).abs() <= bound).all()), (b, L)


EDGES = [0, 1, 2, 7, 15, 16, 17, 31, 33, 47, 63, 64, 65, 129, 511, 513, 2049]


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
@pytest.mark.parametrize("d,G,kvh,ps,gran", [(64, 1, 2, 16, 0), (64, 4, 1, 64, 1), (64, 7, 2, 48, 0), (128, 1, 1, 32, 0),
                                             (128, 2, 3, 16, 1), (128, 4, 2, 64, 0), (128, 7, 2, 128, 1),
                                             (128, 8, 2, 80, 0)])
def test_attention_edges(dtype, d, G, kvh, ps, gran):
    gen = torch.Generator(device="cuda").manual_seed(d + G + ps)
    for lens in (EDGES, [20011]):
        c = make(lens, kvh, G, d, ps, dtype, starts=[(5 * i + 3) % 23 for i in range(len(lens))], gran=gran)
        noise(c, gen)  # slots outside the sequences may hold anything
        x = torch.randn(2, len(lens), max(lens), kvh, d, generator=gen, device="cuda").to(TORCH[dtype])
        x[:, :, ::37] *= 4.0
        ikv.ikv_q4_store(c.shape(), c.cache(max(lens)), c.q4(), 0, 2, x, x.flip(2), c.dense_rows(x), torch.zeros_like(c.len), c.len,
                         max(lens))
        c.pos[torch.rand(c.pos.shape, generator=gen, device="cuda") < 0.2] = -1
        if len(lens) > 9:
            c.pos[8 * (c.rows // len(lens)):9 * (c.rows // len(lens))] = -1  # every slot of a sequence dead
        q = (2.0 * torch.randn(len(lens), G * kvh, d, generator=gen, device="cuda")).to(TORCH[dtype])
        for dead in (False, True):
            cch = c.cache(max(lens), dead_slots=dead)
            n = ikv.ikv_attend_workspace_size(c.shape(), cch)
            ws = torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")  # needs no initialisation
            out = torch.full((len(lens), G * kvh, d), 9.0, dtype=TORCH[dtype], device="cuda")
            score = torch.full((c.rows, c.cap), -7.0, device="cuda")
            ikv.ikv_q4_attend_score(c.shape(), cch, c.q4(), 1, q, out, score, None, 0.0, ws, n)
            assert ikv.ikv_device_status() == 0
            live = c.pos >= 0 if dead else torch.ones_like(c.pos, dtype=torch.bool)
            check(c, 1, q, out, score, dead, live)
            for b, L in enumerate(lens):
                per = c.rows // len(lens)
                assert torch.all(score[b * per:(b + 1) * per, L:] == -7.0)
            # without scores, and once more: the same bits; with a utility: Eq. 4 on the score
            again = torch.full_like(out, 3.0)
            ema = torch.rand(c.rows, c.cap, generator=gen, device="cuda")
            was = ema.clone()
            ikv.ikv_q4_attend_score(c.shape(), cch, c.q4(), 1, q, again, None, None, 0.0, ws, n)
            assert torch.equal(again.view(torch.uint8), out.view(torch.uint8))
            sc2 = torch.full_like(score, -7.0)
            ikv.ikv_q4_attend_score(c.shape(), cch, c.q4(), 1, q, again, sc2, ema, 0.75, ws, n)
            assert torch.equal(again.view(torch.uint8), out.view(torch.uint8)) and torch.equal(sc2, score)
            inside = torch.arange(c.cap, device="cuda")[None] < c.len.repeat_interleave(c.rows // len(lens))[:, None]
            want = torch.where(inside, 0.75 * was + 0.25 * score, was)
            assert bool(((ema - want).abs() <= 2.0 ** -22 * (was.abs() + score.abs())).all())


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
@pytest.mark.parametrize("case", ["growing", "shrinking", "tiny", "zero", "far logits"])
def test_attention_over_uneven_scales(dtype, case):
    """V rows whose sizes span many binades, queries and keys that leave one token everything."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    lens, d, kvh, G = [700, 33], 128, 2, 4
    c = make(lens, kvh, G, d, 64, dtype)
    k = torch.randn(2, 2, 700, kvh, d, generator=gen, device="cuda")
    v = torch.randn(2, 2, 700, kvh, d, generator=gen, device="cuda")
    q = torch.randn(2, G * kvh, d, generator=gen, device="cuda")
    steps = torch.arange(700, device="cuda").view(1, 1, -1, 1, 1) / 700
    if case == "growing":
        v = v * torch.exp2(40 * steps - 20)
    elif case == "shrinking":
        v = v * torch.exp2(20 - 40 * steps)
    elif case == "tiny":
        v, k, q = v * 2.0 ** -100, k * 2.0 ** 30, q * 2.0 ** -30
    elif case == "zero":
        v[:, :, :300] = 0.0
        v[:, 1] = 0.0
        k[:, 1] = 0.0
    else:
        k[:, :, 650:] *= 30.0
        q = q * 8.0
    k, v, q = k.to(TORCH[dtype]), v.to(TORCH[dtype]), q.to(TORCH[dtype])
    ikv.ikv_q4_store(c.shape(), c.cache(700), c.q4(), 0, 2, k, v, c.dense_rows(k), torch.zeros_like(c.len), c.len, 700)
    ws = c.attend_workspace()
    out, score = torch.zeros_like(q), torch.zeros(c.rows, c.cap, device="cuda")
    ikv.ikv_q4_attend_score(c.shape(), c.cache(700), c.q4(), 0, q, out, score, None, 0.0, ws, ws.numel())
    assert ikv.ikv_device_status() == 0
    check(c, 0, q, out, score, False, torch.ones_like(c.pos, dtype=torch.bool))


def test_nan_stays_where_it_is():
    """A NaN group of V makes its 32 channels NaN, one of K its KV head; a dead slot's does nothing."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    for where in ("v", "k", "dead"):
        c = make([100], 2, 4, 64, 16, ikv.IKV_BF16)
        x = torch.randn(2, 1, 100, 2, 64, generator=gen, device="cuda").to(torch.bfloat16)
        k, v = x.clone(), x.clone()
        (k if where == "k" else v)[0, 0, 50, 1, 40] = math.nan
        if where == "dead":
            k[0, 0, 50, 1, 3] = math.inf
            c.pos[0, 50] = -1
        ikv.ikv_q4_store(c.shape(), c.cache(100), c.q4(), 0, 2, k, v, c.dense_rows(k), torch.zeros_like(c.len), c.len, 100)
        q = torch.randn(1, 8, 64, generator=gen, device="cuda").to(torch.bfloat16)
        ws, out = c.attend_workspace(), torch.zeros_like(q)
        ikv.ikv_q4_attend_score(c.shape(), c.cache(100, dead_slots=True), c.q4(), 0, q, out, None, None, 0.0, ws,
                                ws.numel())
        want = torch.zeros(1, 8, 64, dtype=torch.bool, device="cuda")
        if where == "v":
            want[:, 4:, 32:] = True
        elif where == "k":
            want[:, 4:] = True
        assert torch.equal(out.isnan(), want), where


def test_append_streams_and_graphs():
    """Tokens appended one by one (whole steps and layer by layer), on a stream of its own, captured
    in a graph: the same cache as one store of all of them, and the books of ikv_append_token."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    nb, layers, kvh, d, T = 3, 2, 2, 64, 9
    lens = [4, 0, 20]
    new = torch.randn(T, layers, nb, kvh, d, generator=gen, device="cuda").to(torch.bfloat16)
    c = make(lens, kvh, 2, d, 16, ikv.IKV_BF16, room=12, layers=layers)
    c.next_pos.copy_(c.len + 100)
    slot = torch.zeros(nb, dtype=torch.int32, device="cuda")
    buf = new[0].clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    shape, cache, q4 = c.shape(), c.cache(29), c.q4()
    one = ikv.ikv_rows(nb * kvh * d, kvh * d, kvh * d, d, None)
    with torch.cuda.stream(st):
        ikv.ikv_q4_append_token(shape, cache, q4, buf, buf, c.ema, 0, slot, st)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            ikv.ikv_q4_append_token(shape, cache, q4, None, None, c.ema, 0, slot, st)
            for layer in range(layers):
                ikv.ikv_q4_store(shape, cache, q4, layer, 1, buf[layer], buf[layer], one, slot, None, 1, st)
        for t in range(1, T):
            buf.copy_(new[t])
            g.replay()
    st.synchronize()
    assert ikv.ikv_device_status() == 0
    assert c.len.tolist() == [n + T for n in lens] and c.next_pos.tolist() == [n + 100 + T for n in lens]
    assert slot.tolist() == [n + T - 1 for n in lens]
    for b in range(nb):
        assert c.pos[b, lens[b]:lens[b] + T].tolist() == list(range(lens[b] + 100, lens[b] + 100 + T))
        for layer in range(layers):
            for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
                got = values(unpack(paged(c, codes, b, layer, T, lens[b])), paged(c, scale, b, layer, T, lens[b]).double())
                assert torch.equal(got, values(*quantise(new[:, layer, b])))
    # no room left: nothing is stored, slot -1, the error bit
    c.len.copy_(torch.tensor([32, 3, 32], dtype=torch.int32))
    held = [t.clone() for t in c.planes()]
    ikv.ikv_q4_append_token(shape, cache, q4, buf, buf, c.ema, 0, slot)
    assert slot.tolist() == [-1, 3, -1] and c.len.tolist() == [32, 4, 32]
    assert ikv.ikv_device_status() == 4
    for t, was in zip(c.planes(), held):
        for b in (0, 2):
            pages = c.block_table[b].long()
            assert torch.equal(t[:, pages], was[:, pages])


def test_rows_past_four_gigabytes():
    """Code pools of more than 2^32 bytes, the sequence in the last pages of the last layer."""
    d, kvh, ps, pages = 128, 8, 128, 66000
    gen = torch.Generator(device="cuda").manual_seed(9)
    c = Q4Cache(1, 1, 32, kvh, d, 3 * ps, page_size=ps)
    c.num_pages = pages
    c._alloc_pools((1, pages, kvh, ps), "cuda")
    assert c.k.numel() > 2 ** 32
    c.block_table.copy_(torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32))
    c.len.fill_(300)
    x = torch.randn(1, 1, 300, kvh, d, generator=gen, device="cuda").to(torch.bfloat16)
    ikv.ikv_q4_store(c.shape(), c.cache(300), c.q4(), 0, 1, x, x, c.dense_rows(x), torch.zeros_like(c.len), c.len, 300)
    back = [torch.zeros_like(x) for _ in range(2)]
    ikv.ikv_q4_load(c.shape(), c.cache(300), c.q4(), 0, 1, back[0], back[1], c.dense_rows(x), torch.zeros_like(c.len), c.len,
                    300)
    want = values(*quantise(x)).to(torch.bfloat16)
    assert torch.equal(back[0], want) and torch.equal(back[1], want)
    q = torch.randn(1, 32, d, generator=gen, device="cuda").to(torch.bfloat16)
    ws, out, score = c.attend_workspace(), torch.zeros_like(q), torch.zeros(1, c.cap, device="cuda")
    ikv.ikv_q4_attend_score(c.shape(), c.cache(300), c.q4(), 0, q, out, score, None, 0.0, ws, ws.numel())
    assert ikv.ikv_device_status() == 0
    c.pos = torch.zeros(1, c.cap, dtype=torch.int32, device="cuda")
    check(c, 0, q, out, score, False, torch.ones(1, c.cap, dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("lens,kvh,G,gran", [
    ([(7 * i) % 41 for i in range(300)], 8, 4, 0),             # far more units than CTAs, some empty
    ([33] * 200, 4, 7, 1),                                     # as many, of one length
    ([600] * 9, 2, 2, 0),                                      # one length, cut evenly
    ([3000] + [5 + i % 3 for i in range(140)], 2, 8, 0),       # one long among short, two a thread
    ([0] * 130 + [1], 1, 1, 0)])
def test_many_sequences(lens, kvh, G, gran):
    """The deal of the work to the CTAs: batches larger than a CTA, units cut evenly and not."""
    gen = torch.Generator(device="cuda").manual_seed(len(lens))
    d, nb = 64, len(lens)
    c = make(lens, kvh, G, d, 16, ikv.IKV_BF16, starts=[(3 * i) % 19 for i in range(nb)], layers=1, gran=gran, room=20)
    noise(c, gen)
    x = torch.randn(1, nb, max(lens), kvh, d, generator=gen, device="cuda").to(torch.bfloat16)
    ikv.ikv_q4_store(c.shape(), c.cache(max(lens)), c.q4(), 0, 1, x, x.flip(2), c.dense_rows(x), torch.zeros_like(c.len), c.len,
                     max(lens))
    q = (2.0 * torch.randn(nb, G * kvh, d, generator=gen, device="cuda")).to(torch.bfloat16)
    cch = c.cache(max(lens))
    n = ikv.ikv_attend_workspace_size(c.shape(), cch)
    ws = torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")
    out, score = torch.full_like(q, 9.0), torch.full((c.rows, c.cap), -7.0, device="cuda")
    ikv.ikv_q4_attend_score(c.shape(), cch, c.q4(), 0, q, out, score, None, 0.0, ws, n)
    assert ikv.ikv_device_status() == 0
    check(c, 0, q, out, score, False, torch.ones_like(c.pos, dtype=torch.bool))


@pytest.mark.parametrize("lens,kvh,G,d,dtype", [([3000], 1, 8, 128, ikv.IKV_F32), ([40, 900, 0, 17], 4, 7, 128, ikv.IKV_BF16),
                                                ([250] * 40, 2, 1, 64, ikv.IKV_BF16)])
def test_nothing_written_outside_the_buffers(lens, kvh, G, d, dtype):
    """Patterns behind the workspace, around the outputs and in the pools stay as they were."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    c = make(lens, kvh, G, d, 16, dtype, layers=1)
    noise(c, gen)
    x = torch.randn(1, len(lens), max(lens), kvh, d, generator=gen, device="cuda").to(TORCH[dtype])
    ikv.ikv_q4_store(c.shape(), c.cache(max(lens)), c.q4(), 0, 1, x, x, c.dense_rows(x), torch.zeros_like(c.len), c.len, max(lens))
    pools = [t.clone() for t in c.planes()]
    n = ikv.ikv_attend_workspace_size(c.shape(), c.cache(max(lens)))
    ws = torch.full((n + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
    q = torch.randn(len(lens), G * kvh, d, generator=gen, device="cuda").to(TORCH[dtype])
    out = torch.full((len(lens) + 2, G * kvh, d), 5.0, dtype=TORCH[dtype], device="cuda")
    score = torch.full((c.rows + 2, c.cap), 5.0, device="cuda")
    ema = torch.full((c.rows + 2, c.cap), 5.0, device="cuda")
    ikv.ikv_q4_attend_score(c.shape(), c.cache(max(lens)), c.q4(), 0, q, out[1:-1], score[1:-1], ema[1:-1], 0.5, ws, n)
    assert ikv.ikv_device_status() == 0
    assert bool((ws[n:] == 0x5A).all())
    for t in (out, score, ema):
        assert bool((t[0] == 5.0).all()) and bool((t[-1] == 5.0).all())
    for t, was in zip(c.planes(), pools):
        assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
    check(c, 0, q, out[1:-1], score[1:-1], False, torch.ones_like(c.pos, dtype=torch.bool))


@pytest.mark.parametrize("kvh,G,gran,dtype", [(2, 4, 1, ikv.IKV_BF16), (2, 2, 0, ikv.IKV_F32), (1, 7, 0, ikv.IKV_BF16)])
@pytest.mark.parametrize("nb", [80, 160])
def test_scores_of_many_tokens(kvh, G, gran, dtype, nb):
    """Score passes whose threads take four tokens, one block of them or several, against one token a thread."""
    gen = torch.Generator(device="cuda").manual_seed(nb + G)
    d = 64
    lens = [(37 * i) % 90 for i in range(nb)]
    lens[3], lens[nb // 2], lens[nb - 1] = 4601, 2049, 4095
    c = make(lens, kvh, G, d, 16, dtype, starts=[(3 * i) % 19 for i in range(nb)], layers=1, gran=gran, room=20)
    noise(c, gen)
    dt = torch.float32 if dtype == ikv.IKV_F32 else torch.bfloat16
    x = torch.randn(1, nb, max(lens), kvh, d, generator=gen, device="cuda").to(dt)
    ikv.ikv_q4_store(c.shape(), c.cache(max(lens)), c.q4(), 0, 1, x, x.flip(2), c.dense_rows(x), torch.zeros_like(c.len), c.len,
                     max(lens))
    live = torch.rand(c.pos.shape, generator=gen, device="cuda") > 0.3
    c.pos.copy_(torch.where(live, c.pos, -1 - c.pos))
    q = (2.0 * torch.randn(nb, G * kvh, d, generator=gen, device="cuda")).to(dt)
    cch = c.cache(max(lens), dead_slots=True)
    n = ikv.ikv_attend_workspace_size(c.shape(), cch)
    ws = torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 9.0)
    was = torch.rand(c.rows, c.cap, generator=gen, device="cuda")
    got = []
    for shift in (0, 1):  # the second lies off the 16-byte boundaries
        score = torch.full((c.rows * c.cap + 4,), -7.0, device="cuda")
        ema = torch.zeros(c.rows * c.cap + 4, device="cuda")
        inner = slice(shift, shift + c.rows * c.cap)
        ema[inner] = was.flatten()
        ikv.ikv_q4_attend_score(c.shape(), cch, c.q4(), 0, q, out, score[inner], ema[inner], 0.75, ws, n)
        assert ikv.ikv_device_status() == 0
        outside = torch.ones_like(score, dtype=torch.bool)
        outside[inner] = False
        assert bool((score[outside] == -7.0).all()) and bool((ema[outside] == 0.0).all())
        got.append((score[inner].view(c.rows, c.cap), ema[inner].view(c.rows, c.cap)))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    score, ema = got[0]
    check(c, 0, q, out, score, True, live)
    inside = torch.arange(c.cap, device="cuda") < c.len.repeat_interleave(c.rows // nb)[:, None]
    assert bool((score[~inside] == -7.0).all()) and torch.equal(ema[~inside], was[~inside])
    # (two products and a sum, each rounded)
    want = 0.75 * was.double() + 0.25 * score.double()
    assert bool(((ema.double() - want).abs() <= want * 2.0 ** -22)[inside].all())
