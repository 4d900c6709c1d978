"""A NaN or infinite logit leaves no number in its heads' outputs, in however many parts the attention
computes them: the sum of their weights is NaN, which is not the sum of a sequence without live slots."""
import math

import pytest
import torch

from paper_2609_03515_gb300 import DecodeCache, Q4Cache, ikv

pytestmark = pytest.mark.gpu

DT = {ikv.IKV_F32: torch.float32, ikv.IKV_BF16: torch.bfloat16}


def _cache(cls, lens, kvh, G, d, dtype):
    c = cls(len(lens), 1, G * kvh, kvh, d, max(lens) + 8, dtype=dtype, page_size=16, page_perm_seed=2)
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    return c


def _check(out, lens, G, what, at):
    """NaN in sequence at: every head's output (query) or those of KV head 1 (key)."""
    want = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    want[at, (G if what == "key" else 0):] = True
    assert torch.equal(out.isnan(), want)
    for b, L in enumerate(lens):
        if L == 0:
            assert not out[b].any()


# units of one segment, of 2, of 5, of 40, one of many among units of one, a batch of several each
LENS = [[100], [200], [600], [5000], [5000] + [20] * 15, [0, 3000, 2500, 2900] * 4]


@pytest.mark.parametrize("what", ["key", "query"])
@pytest.mark.parametrize("dtype,d", [(ikv.IKV_F32, 64), (ikv.IKV_BF16, 128)])
@pytest.mark.parametrize("lens", LENS)
def test_four_bit_attention(lens, dtype, d, what):
    kvh, G, dt = 2, 4, DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(d)
    c = _cache(Q4Cache, lens, kvh, G, d, dtype)
    b = max(range(len(lens)), key=lambda i: lens[i])
    x = torch.randn(1, len(lens), max(lens), kvh, d, generator=gen, device="cuda").to(dt)
    v = x.flip(2).contiguous()
    q = torch.randn(len(lens), G * kvh, d, generator=gen, device="cuda").to(dt)
    if what == "key":
        x[0, b, lens[b] // 2, 1, 3] = math.nan
    else:
        q[b, :, 5] = math.inf
    ikv.ikv_q4_store(c.shape(), c.cache(max(lens)), c.q4(), 0, 1, x, v, c.dense_rows(x), torch.zeros_like(c.len), c.len, max(lens))
    ws = c.attend_workspace()
    out, score = torch.full_like(q, 7.0), torch.zeros(c.rows, c.cap, device="cuda")
    ikv.ikv_q4_attend_score(c.shape(), c.cache(max(lens)), c.q4(), 0, q, out, score, None, 0.0, ws, ws.numel())
    assert ikv.ikv_device_status() == 0
    _check(out, lens, G, what, b)
    for i, L in enumerate(lens):
        assert bool(score[i, :L].isnan().all()) == (i == b or L == 0)


@pytest.mark.parametrize("what", ["key", "query"])
@pytest.mark.parametrize("dtype,d", [(ikv.IKV_F32, 64), (ikv.IKV_F32, 128), (ikv.IKV_BF16, 64), (ikv.IKV_BF16, 128)])
@pytest.mark.parametrize("lens", LENS + [[5000] * 64])
def test_dense_attention(lens, dtype, d, what):
    kvh, G, dt = 2, 4, DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(d)
    c = _cache(DecodeCache, lens, kvh, G, d, dtype)
    c.k.normal_(generator=gen)
    c.v.normal_(generator=gen)
    b = max(range(len(lens)), key=lambda i: lens[i])
    q = torch.randn(len(lens), G * kvh, d, generator=gen, device="cuda").to(dt)
    if what == "key":
        s = lens[b] // 2
        c.k[0, int(c.block_table[b, s // 16]), 1, s % 16, 3] = math.nan
    else:
        q[b, :, 5] = math.nan
    cache = c.cache(max(lens))
    n = ikv.ikv_attend_workspace_size(c.shape(), cache)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    out, score = torch.full_like(q, 7.0), torch.zeros(c.rows, c.cap, device="cuda")
    ikv.ikv_decode_attend_score(c.shape(), cache, 0, q, out, score, None, 0.0, ws, n)
    assert ikv.ikv_device_status() == 0
    _check(out, lens, G, what, b)
