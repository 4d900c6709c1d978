"""Block table entries that name no page: every page call that meets one reports it and counts nothing for it."""
import pytest
import torch

from paper_2609_03515_gb300 import DecodeCache, ikv

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pool(nb=2, cap=64, pages=12):
    """Sequence 0 holds three pages of 16 slots."""
    c = DecodeCache(nb, 1, 1, 1, 64, cap, page_size=16, pool_pages=pages)
    ws = c.pages_workspace()
    ikv.ikv_pages_writable(c.shape(), c.cache(0), c.pages(), None, i32([48] + [0] * (nb - 1)), 48, None, ws, ws.numel())
    c.len[0] = 48
    c.k.normal_()
    assert ikv.ikv_device_status() == 0
    return c, ws


@pytest.mark.parametrize("bad", [-1, 13, 1 << 30])
def test_release_and_fork(bad):
    c, _ = pool()
    c.block_table[0, 1] = bad
    refs = c.refs.clone()
    ikv.ikv_pages_fork(c.shape(), c.cache(0), c.pages(), 1, i32([0]), i32([1]), None)
    assert ikv.ikv_device_status() == 128
    assert c.block_table.tolist() == [[1, bad, 3, 0], [1, 0, 3, 0]]  # (what is no page is not passed on)
    c.len.zero_()
    ikv.ikv_pages_release(c.shape(), c.cache(0), c.pages(), 0)
    assert ikv.ikv_device_status() == 128
    assert c.block_table.tolist() == [[0, bad, 0, 0], [0, 0, 0, 0]]
    refs[1] -= 1
    refs[3] -= 1
    assert torch.equal(c.refs, refs)


@pytest.mark.parametrize("bad", [-1, 13, 1 << 30])
@pytest.mark.parametrize("nb,cap", [(2, 64), (2100, 64)])  # tables that the plan writes, and too many entries for it
def test_compaction(bad, nb, cap):
    c, ws = pool(nb, cap)
    c.block_table[0, 3] = bad  # behind the last slot: nothing is read from it
    keep = torch.arange(c.cap, dtype=torch.int32, device="cuda").repeat(nb, 1)
    ikv.ikv_pages_compact(c.shape(), c.cache(0), c.pages(), keep, i32([20] + [-1] * (nb - 1)), None, None, ws, ws.numel())
    assert ikv.ikv_device_status() == 128
    assert c.block_table[0].tolist() == [1, 2, 0, 0] and c.refs.tolist() == [1, 1, 1] + [0] * 10
