"""What the workspaces of the shared-prefix and window calls hold room for."""
import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_03515_gb300 import ikv

    return ikv


def _sizes(lib, dtype, page, dead):
    shape = lib.ikv_shape(batch=8, layers=2, q_heads=8, kv_heads=2, head_dim=128, dtype=dtype,
                          granularity=lib.IKV_GRAN_KVHEAD)
    pages = (1 << 20) // page
    cache = lib.ikv_cache(k=16, v=16, block_table=16, num_pages=4, page_size=page, max_pages=pages, len=16, pos=16,
                          next_pos=16, max_len=100, dead_slots=dead)
    window = lib.ikv_window(100, 4, None, None, 3, 0, 0)
    prefix = lib.ikv_prefix(1, 16, 16, 16)
    return lib.ikv_window_workspace_size(shape, cache, window), lib.ikv_prefix_workspace_size(shape, cache, prefix)


def test_live_slots_as_bits_only_where_they_are_read(lib):
    """The kernels on the tensor cores read a bit a slot, the others the positions."""
    for dtype, page in ((lib.IKV_F32, 16), (lib.IKV_F32, 64), (lib.IKV_BF16, 20)):
        assert _sizes(lib, dtype, page, 1) == _sizes(lib, dtype, page, 0)
    bits = 8 * 2 * (1 << 20) // 8
    for x, y in zip(_sizes(lib, lib.IKV_BF16, 64, 1), _sizes(lib, lib.IKV_BF16, 64, 0)):
        assert x - y == bits
