"""Pages as large as the page calls take: a compaction whose rows of one plane pass 2^31 words."""
import pytest
import torch

from paper_2609_03515_gb300 import ikv

pytestmark = pytest.mark.gpu


def test_compaction_of_pages_of_16_mb_a_head():
    heads, row, pages = 256, (1 << 22) - 1, 6  # a page of one slot: 4.3 GB over its heads
    ids = torch.arange(pages * heads, dtype=torch.int32, device="cuda").view(1, pages, heads, 1, 1)
    col = torch.arange(row, dtype=torch.int32, device="cuda")
    plane = torch.empty(1, pages, heads, 1, row, dtype=torch.int32, device="cuda")
    plane.copy_((ids << 20).expand_as(plane)).add_(col >> 2)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, refs, length, pos = i32([[1, 2, 3]]), i32([1, 1, 1, 1, 0, 0]), i32([3]), i32([[0, 1, 2]])
    shape = ikv.ikv_shape(1, 1, heads, heads, 64, ikv.IKV_BF16, ikv.IKV_GRAN_SEQ)
    cache = ikv.ikv_cache(plane.data_ptr(), plane.data_ptr(), table.data_ptr(), pages, 1, 3, length.data_ptr(), pos.data_ptr(),
                          None, 3)
    pool = ikv.ikv_pages_of(refs, [plane])
    n = ikv.ikv_pages_workspace_size(shape, cache, pool)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    ikv.ikv_pages_compact(shape, cache, pool, i32([[1, 2, 0]]), i32([2]), None, None, ws, n)
    assert ikv.ikv_device_status() == 0
    assert table.tolist() == [[4, 5, 0]] and refs.tolist() == [1, 0, 0, 0, 1, 1] and pos[0, :2].tolist() == [1, 2]
    for page, was in ((4, 2), (5, 3)):
        for h in range(0, heads, 8):
            want = (ids[0, was, h:h + 8, 0] << 20) + (col >> 2)
            assert torch.equal(plane[0, page, h:h + 8, 0], want)
