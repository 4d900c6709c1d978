"""The bounded waits of the shared-prefix and window attentions: a launch whose wait runs out reports it, leaves
scores and utilities whole, and the next launch is right."""
import pytest
import torch

from paper_2609_03515_gb300 import ikv
from rows_ref import DT, MARK, Cache
from test_gpu_prefix import Call, reference

pytestmark = pytest.mark.gpu


def make(d=128):
    lens = [500, 470, 480, 300, 90]
    c = Cache(lens, 4, 4, d, "bf16", 64, seed=21, share=[(0, [1, 2], 460)]).device()
    return Call(c, [[0, 1, 2]], [460], ema=True)


def same(call):
    """The marked places only: nothing was stored."""
    assert bool((call.score == MARK).all())
    assert torch.equal(call.ema.cpu(), call.ema0)


def right(call):
    out, tol, score, stol = reference(call)
    assert bool(((call.out.cpu().double() - out).abs() <= tol).all())
    for b, n in enumerate(call.c.lens):
        assert bool(((call.score[b, :n].cpu().double() - score[b, :n]).abs() <= stol[b, :n]).all())
        want = call.alpha * call.ema0[b, :n].double() + (1 - call.alpha) * score[b, :n]
        # two products and a sum in 32 bits
        assert bool(((call.ema[b, :n].cpu().double() - want).abs() <= stol[b, :n] + 4 * 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("d", [64, 128])
def test_prefix_attention_that_gives_up_leaves_scores_and_utilities(d):
    call = make(d)
    call.ws.fill_(0x7F)  # (parts that were never written would be large numbers)
    ikv.ikv_test_stall_next_attention()
    call.run()
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 1
    assert ikv.ikv_device_status() == 0
    same(call)
    call.run()
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 0
    right(call)


@pytest.mark.parametrize("d", [64, 128])
def test_score_pass_that_gives_up_stores_no_partial_sums(d):
    """It stops between the KV heads of an item: sums over the first alone must not be stored."""
    call = make(d)
    ikv.ikv_test_stall_next_score()
    call.run()
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 1
    assert ikv.ikv_device_status() == 0
    same(call)
    out, tol, _, _ = reference(call)
    assert bool(((call.out.cpu().double() - out).abs() <= tol).all())
    call.run()
    torch.cuda.synchronize()
    assert ikv.ikv_device_status() == 0
    right(call)


def test_window_that_gives_up_reports_it_and_the_next_call_is_right():
    c = Cache([700, 33], 2, 4, 128, "bf16", 16, seed=22, layers=1).device()
    q = torch.randn(733, c.h * c.d, generator=torch.Generator().manual_seed(3)).to(DT["bf16"]).cuda()
    count = torch.tensor([700, 33], dtype=torch.int32).cuda()
    row0 = torch.tensor([0, 700], dtype=torch.int32).cuda()
    win = ikv.ikv_window(100, 4, row0.data_ptr(), count.data_ptr(), 700, 0, 0)
    n = ikv.ikv_window_workspace_size(c.shape(), c.cache(), win)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    first, again = torch.empty_like(q), torch.full_like(q, MARK)

    def call(out):
        ikv.ikv_window_attend(c.shape(), c.cache(), win, 0, q, out, ws, n)
        torch.cuda.synchronize()
        return ikv.ikv_device_status()

    assert call(first) == 0
    ikv.ikv_test_stall_next_attention()
    assert call(again) == 1
    again.fill_(MARK)
    assert call(again) == 0
    assert torch.equal(first, again)
