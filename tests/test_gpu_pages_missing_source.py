"""Compactions that are told to keep a slot without a page."""
import pytest
import torch

from paper_2609_03515_gb300 import DecodeCache, ikv

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("gran", [ikv.IKV_GRAN_SEQ, ikv.IKV_GRAN_KVHEAD])
def test_a_kept_slot_without_a_page(gran):
    """It is reported, nothing is copied out of page 0, and the other slots move as they should."""
    c = DecodeCache(1, 1, 2, 2, 64, 64, page_size=16, pool_pages=9, granularity=gran)
    shape, cache, pages, ws = c.shape(), c.cache(0), c.pages(), c.pages_workspace()
    ikv.ikv_pages_writable(shape, cache, pages, None, i32([48]), 48, None, ws, ws.numel())
    c.len.fill_(48)
    for t in c.planes():
        t.copy_(torch.arange(t.numel(), device="cuda").view(t.shape) % 251)
    before = [t.clone() for t in c.planes()]
    c.block_table[0, 1] = 0  # slots 16 .. 31
    keep = torch.zeros(c.rows, c.cap, dtype=torch.int32, device="cuda")
    kept = list(range(4, 10)) + list(range(20, 24)) + list(range(40, 48))
    keep[:, :len(kept)] = i32(kept)
    ikv.ikv_pages_compact(shape, cache, pages, keep, i32([len(kept)] * c.rows), None, None, ws, ws.numel())
    assert ikv.ikv_device_status() == 128
    assert c.len.tolist() == [len(kept)] and c.block_table.tolist() == [[4, 5, 0, 0]]
    for t, was in zip(c.planes(), before):
        for j, slot in enumerate(kept):
            new = t[0, 4 + j // 16, :, j % 16]
            if 16 <= slot < 32:
                assert torch.equal(new, was[0, 4 + j // 16, :, j % 16])  # as the fresh page was
            else:
                assert torch.equal(new, was[0, 1 + slot // 16, :, slot % 16])
