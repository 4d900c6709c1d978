"""The 4-bit attention over all the sizes that its scales can have, against plain fp64.

Weights and their sums do not depend on V, so the scores' bound is that of their own roundings whatever
V holds, and the outputs' bound is kept group of channels by group.  The roundings:
  a logit: products of codes and queries are exact and summed in fp32 by the tensor unit, at most
  2^-18 of the sum of the terms' magnitudes (which each test keeps small);
  a probability: 2^-22 for the exponential, 2^-21 for its argument (of some tens), sums in fp32 over at
  most 2^4 terms a lane and as many lanes, warps and segments: 2^-19 in all;
  an output: its weights are rounded to 2^-11 of each (bf16) or 2^-22 (fp32), or, far below the
  largest, to 2^-25 or 2^-36 with the group's largest scale seen at 2^4 or above and the largest
  weight's p at 1 or above; products are summed in fp32: 2^-19; a bf16 output is rounded
  once more (2^-8 covers it)."""
import math

import pytest
import torch
from test_gpu_q4 import TORCH, make, paged, unpack, values

from paper_2609_03515_gb300 import ikv

pytestmark = pytest.mark.gpu


def attend(c, q, most):
    ws = c.attend_workspace()
    out, score = torch.zeros_like(q), torch.zeros(c.rows, c.cap, device="cuda")
    ikv.ikv_q4_attend_score(c.shape(), c.cache(most), c.q4(), 0, q, out, score, None, 0.0, ws, ws.numel())
    assert ikv.ikv_device_status() == 0
    return out, score


def check(c, q, out, score):
    two, G, D = c.dtype == ikv.IKV_F32, c.q_heads // c.kv_heads, c.head_dim
    for b, L in enumerate(c.len.tolist()):
        pooled, zmax = torch.zeros(L, dtype=torch.float64, device="cuda"), 0.0
        for g in range(c.kv_heads):
            K = values(unpack(paged(c, c.k, b, 0, L))[:, g], paged(c, c.k_scale, b, 0, L)[:, g].double())
            s = paged(c, c.v_scale, b, 0, L)[:, g].double()
            V = values(unpack(paged(c, c.v, b, 0, L))[:, g], s)
            x = q[b, g * G:(g + 1) * G].double()
            p = torch.softmax(x @ K.T / math.sqrt(D), -1)
            zmag = float((x.abs() @ K.abs().T / math.sqrt(D)).amax())
            zmax = max(zmax, zmag)
            pooled += p.sum(0) / c.q_heads
            o, mag = p @ V, p @ V.abs()
            one = (2.0 ** -21 if two else 2.0 ** -10) + zmag * 2.0 ** -18 + 2.0 ** -19
            small = L * 2.0 ** (-36 if two else -25) * 6.0 / 16 * s.amax(0).repeat_interleave(32)
            bound = mag * one + small + (0.0 if two else o.abs() * 2.0 ** -8) + 2.0 ** -149
            err = (out[b, g * G:(g + 1) * G].double() - o).abs()
            assert bool((err <= bound).all()), (b, g, float((err / bound).max()))
        err = (score[b, :L].double() - pooled).abs()
        assert bool((err <= pooled * (zmax * 2.0 ** -18 + 2.0 ** -19) + 2.0 ** -126).all()), (b, float((err / pooled).max()))


SIZES = ["2^100", "2^118", "2^122", "2^-60", "2^-112", "tiny then large", "large then tiny", "groups apart", "one group large",
         "one group zero", "all binades"]


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
@pytest.mark.parametrize("d,G", [(128, 4), (128, 7), (64, 2), (64, 8)])
@pytest.mark.parametrize("case", SIZES)
def test_sizes_of_values(dtype, d, G, case):
    """V over the whole range of its format, with logits that differ by some 15 log2 units; units of one
    segment and of several."""
    gen = torch.Generator(device="cuda").manual_seed(d + G)
    lens, kvh = [50, 900, 333], 2
    n, most = len(lens), max(lens)
    c = make(lens, kvh, G, d, 64, dtype, layers=1)
    shape = (1, n, most, kvh, d)
    k = torch.randn(shape, generator=gen, device="cuda")
    v = torch.randn(shape, generator=gen, device="cuda").clamp(-6, 6)
    v = v + 0.75 * v.sign()  # (outputs that do not vanish)
    q = 2.0 * torch.randn(n, G * kvh, d, generator=gen, device="cuda")
    at = (torch.arange(most, device="cuda") / most).view(1, 1, -1, 1, 1)
    group = (torch.arange(d, device="cuda") // 32).double()
    power = torch.zeros(shape, dtype=torch.float64, device="cuda")
    if case.startswith("2^"):
        power += float(case[2:])
    elif case == "tiny then large":
        power += torch.where(at < 0.5, -100.0, 60.0)
    elif case == "large then tiny":
        power += torch.where(at < 0.01, 60.0, -100.0)
    elif case == "groups apart":
        power += 40.0 - 60.0 * group
    elif case == "one group large":
        power += torch.where(group == 1, 110.0, -20.0)
    elif case == "one group zero":
        power += torch.where(group == 0, -130.0, 3.0)
    else:
        power += -110.0 + 225.0 * ((at * 7) % 1.0)
    v = (v.double() * torch.exp2(power)).float()
    k, v, q = k.to(TORCH[dtype]), v.to(TORCH[dtype]), q.to(TORCH[dtype])
    ikv.ikv_q4_store(c.shape(), c.cache(most), c.q4(), 0, 1, k, v, c.dense_rows(k), torch.zeros_like(c.len), c.len, most)
    out, score = attend(c, q, most)
    check(c, q, out, score)


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
def test_scores_do_not_depend_on_values(dtype):
    """The same queries and keys over values of any size: the same scores, bit for bit."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    lens, kvh, G, d = [2100, 70], 2, 4, 128
    c = make(lens, kvh, G, d, 64, dtype, layers=1)
    k = torch.randn(1, 2, 2100, kvh, d, generator=gen, device="cuda").to(TORCH[dtype])
    q = (2.0 * torch.randn(2, G * kvh, d, generator=gen, device="cuda")).to(TORCH[dtype])
    got = []
    for e in (0, -60, -118, 124, None):
        v = torch.randn(k.shape, generator=gen, device="cuda").clamp(-4, 4)
        v = (v * 2.0 ** e if e is not None else v * torch.exp2(torch.randint(-100, 100, (2100, 1, 1), generator=gen, device="cuda").float())).to(k.dtype)
        ikv.ikv_q4_store(c.shape(), c.cache(2100), c.q4(), 0, 1, k, v, c.dense_rows(k), torch.zeros_like(c.len), c.len, 2100)
        got.append(attend(c, q, 2100)[1])
    assert all(torch.equal(got[0], x) for x in got[1:])


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
@pytest.mark.parametrize("lens", [[40], [900], [9000], [40000], [300] * 30])
def test_largest_values_do_not_overflow(dtype, lens):
    """Equal weights over values of the format's largest size: their mean, however many there are."""
    kvh, G, d = 1, 4, 64
    c = make(lens, kvh, G, d, 64, dtype, layers=1)
    v = torch.full((1, len(lens), max(lens), kvh, d), 1.5 * 2.0 ** 125, device="cuda").to(TORCH[dtype])
    k = torch.zeros_like(v)
    q = torch.ones(len(lens), G * kvh, d, device="cuda").to(TORCH[dtype])
    ikv.ikv_q4_store(c.shape(), c.cache(max(lens)), c.q4(), 0, 1, k, v, c.dense_rows(k), torch.zeros_like(c.len), c.len, max(lens))
    out, _ = attend(c, q, max(lens))
    # (6 s of a scale s = 2^123 exactly; sums of equal terms: 2^-18)
    assert bool(((out.double() / (1.5 * 2.0 ** 125) - 1).abs() <= 2.0 ** -18).all())


@pytest.mark.parametrize("dtype", [ikv.IKV_F32, ikv.IKV_BF16])
@pytest.mark.parametrize("n", [1, 2, 60, 700, 3000])
def test_equal_keys_score_alike(dtype, n):
    """Tokens whose keys are alike get 1 / n each, however large their logits: the sum of the weights and a
    token's probability go by the same logit, so its roundings cancel and two exponentials (2^-22
    each) and the sum (at most 2^4 terms a lane, 2^-21) remain."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    nb, kvh, G, d = 24, 1, 1, 64
    c = make([n] * nb, kvh, G, d, 64, dtype, layers=1)
    k = torch.randn(1, nb, 1, kvh, d, generator=gen, device="cuda")
    q = torch.randn(nb, G * kvh, d, generator=gen, device="cuda")
    q = (q * torch.linspace(0.1, 12, nb, device="cuda").view(-1, 1, 1) + 3.0 * k[0, :, 0].repeat_interleave(G, 1)).to(TORCH[dtype])
    k = k.expand(-1, -1, n, -1, -1).to(TORCH[dtype]).contiguous()
    v = torch.randn(k.shape, generator=gen, device="cuda").to(TORCH[dtype])
    ikv.ikv_q4_store(c.shape(), c.cache(n), c.q4(), 0, 1, k, v, c.dense_rows(k), torch.zeros_like(c.len), c.len, n)
    _, score = attend(c, q, n)
    err = (score[:, :n].double() * n - 1).abs()
    assert bool((err <= 2.0 ** -20).all()), float(err.max())


def test_many_query_heads():
    """As many heads as a row's references and sums take more than 48 KB of shared memory for."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    kvh, G, d = 600, 8, 64
    c = make([70], kvh, G, d, 16, ikv.IKV_BF16, layers=1, room=2)
    k = torch.randn(1, 1, 70, kvh, d, generator=gen, device="cuda").to(torch.bfloat16)
    q = torch.randn(1, G * kvh, d, generator=gen, device="cuda").to(torch.bfloat16)
    ikv.ikv_q4_store(c.shape(), c.cache(70), c.q4(), 0, 1, k, k.flip(2).contiguous(), c.dense_rows(k), torch.zeros_like(c.len), c.len, 70)
    out, score = attend(c, q, 70)
    check(c, q, out, score)
