"""Refusals of the 4-bit cache and page pool entry points, on the host before any launch."""
import ctypes

import pytest
import torch

from paper_2609_03515_gb300 import Q4Cache, ikv

A = 64  # an address on a 16-byte boundary, never read


def shape(**kw):
    d = dict(batch=2, layers=3, q_heads=8, kv_heads=2, head_dim=64, dtype=ikv.IKV_BF16, granularity=ikv.IKV_GRAN_SEQ)
    d.update(kw)
    return ikv.ikv_shape(**d)


def cache(**kw):
    d = dict(k=A, v=A, block_table=A, num_pages=9, page_size=16, max_pages=4, len=A, pos=A, next_pos=A, max_len=60)
    d.update(kw)
    return ikv.ikv_cache(**d)


def pages(**kw):
    p = ikv.ikv_pages()
    p.refs, p.n_planes = A, 2
    for i in range(4):
        p.plane[i], p.row_bytes[i] = A, 128
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[v[0]] = v[1]
        else:
            setattr(p, k, v)
    return p


def rows(**kw):
    d = dict(layer=1024, seq=512, token=128, head=64, row0=None)
    d.update(kw)
    return ikv.ikv_rows(**d)


def status(name, *args):
    st = ikv.raw_status(name, *[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args])
    assert ikv.ikv_last_error() != ""
    return st


Q4 = ikv.ikv_q4(A, A)
COMMON = [
    (shape(head_dim=96), cache(), Q4, ikv.IKV_ERR_UNSUPPORTED),
    (shape(q_heads=6), cache(), Q4, ikv.IKV_ERR_UNSUPPORTED),
    (shape(dtype=5), cache(), Q4, ikv.IKV_ERR_ARG),
    (shape(batch=0), cache(), Q4, ikv.IKV_ERR_SHAPE),
    (shape(), cache(page_size=24), Q4, ikv.IKV_ERR_UNSUPPORTED),
    (shape(), cache(page_size=8), Q4, ikv.IKV_ERR_SHAPE),  # max_len 60 > cap 32 comes first
    (shape(), cache(page_size=8, max_pages=8), Q4, ikv.IKV_ERR_UNSUPPORTED),
    (shape(), cache(k=None), Q4, ikv.IKV_ERR_ARG),
    (shape(), cache(k=A + 8), Q4, ikv.IKV_ERR_ALIGN),
    (shape(), cache(max_len=65), Q4, ikv.IKV_ERR_SHAPE),
    (shape(), cache(dead_slots=1, pos=None), Q4, ikv.IKV_ERR_ARG),
    (shape(), cache(), ikv.ikv_q4(None, A), ikv.IKV_ERR_ARG),
    (shape(), cache(), ikv.ikv_q4(A, A + 2), ikv.IKV_ERR_ALIGN),
]


@pytest.mark.parametrize("i", range(len(COMMON)))
def test_shapes_and_caches(i):
    s, c, q, want = COMMON[i]
    for name in ("ikv_q4_store", "ikv_q4_load"):
        assert status(name, s, c, q, 0, 1, A, A, rows(), None, None, 1, None) == want
    assert status("ikv_q4_attend_score", s, c, q, 0, A, A, None, None, ctypes.c_float(0), A, 1 << 30, None) == want
    assert status("ikv_q4_append_token", s, c, q, A, A, None, 0, A, None) == want


@pytest.mark.parametrize("layer0,n,k,r,most,want", [
    (-1, 1, A, rows(), 1, ikv.IKV_ERR_ARG), (0, 4, A, rows(), 1, ikv.IKV_ERR_ARG), (3, 1, A, rows(), 1, ikv.IKV_ERR_ARG),
    (0, -1, A, rows(), 1, ikv.IKV_ERR_ARG), (0, 1, None, rows(), 1, ikv.IKV_ERR_ARG),
    (0, 1, A + 8, rows(), 1, ikv.IKV_ERR_ALIGN), (0, 1, A, rows(token=132), 1, ikv.IKV_ERR_ALIGN),
    (0, 1, A, rows(head=68), 1, ikv.IKV_ERR_ALIGN), (0, 1, A, rows(layer=3), 1, ikv.IKV_ERR_ALIGN),
    (0, 1, A, rows(seq=-4), 1, ikv.IKV_ERR_ALIGN), (0, 1, A, rows(), -1, ikv.IKV_ERR_SHAPE),
    (0, 1, A, rows(), 65, ikv.IKV_ERR_SHAPE)])
def test_store_and_load(layer0, n, k, r, most, want):
    for name in ("ikv_q4_store", "ikv_q4_load"):
        assert status(name, shape(), cache(), Q4, layer0, n, k, A, r, None, None, most, None) == want
    assert ikv.raw_status("ikv_q4_store", None, None, None, 0, 1, A, A, None, None, None, 1, None) == ikv.IKV_ERR_ARG


def test_attend():
    def call(layer=0, q=A, out=A, ema=None, alpha=0.5, ws=A, n=1 << 30):
        return status("ikv_q4_attend_score", shape(), cache(), Q4, layer, q, out, None, ema, ctypes.c_float(alpha), ws,
                      ctypes.c_size_t(n), None)

    assert call(layer=3) == ikv.IKV_ERR_ARG and call(layer=-1) == ikv.IKV_ERR_ARG
    assert call(q=None) == ikv.IKV_ERR_ARG and call(out=A + 4) == ikv.IKV_ERR_ALIGN
    assert call(ema=A, alpha=1.5) == ikv.IKV_ERR_ARG and call(ema=A, alpha=float("nan")) == ikv.IKV_ERR_ARG
    assert call(ws=None) == ikv.IKV_ERR_WORKSPACE and call(n=100) == ikv.IKV_ERR_WORKSPACE
    assert call(ws=A + 4) == ikv.IKV_ERR_ALIGN


def test_append():
    def call(c, k=A, v=A, slot=A):
        return status("ikv_q4_append_token", shape(), c, Q4, k, v, None, 0, slot, None)

    assert call(cache(), slot=None) == ikv.IKV_ERR_ARG
    assert call(cache(), v=None) == ikv.IKV_ERR_ARG and call(cache(), k=None) == ikv.IKV_ERR_ARG
    assert call(cache(), k=A + 2) == ikv.IKV_ERR_ALIGN
    assert call(cache(next_pos=None)) == ikv.IKV_ERR_ARG
    assert call(cache(max_len=64)) == ikv.IKV_ERR_SHAPE


PAGES = [
    (shape(kv_heads=3), cache(), pages(), ikv.IKV_ERR_SHAPE),
    (shape(), cache(len=None), pages(), ikv.IKV_ERR_ARG),
    (shape(), cache(), pages(refs=None), ikv.IKV_ERR_ARG),
    (shape(), cache(), pages(n_planes=0), ikv.IKV_ERR_SHAPE),
    (shape(), cache(), pages(n_planes=5), ikv.IKV_ERR_SHAPE),
    (shape(), cache(), pages(plane=(1, None)), ikv.IKV_ERR_ARG),
    (shape(), cache(), pages(plane=(1, A + 4)), ikv.IKV_ERR_ALIGN),
    (shape(), cache(), pages(row_bytes=(0, 0)), ikv.IKV_ERR_SHAPE),
    (shape(), cache(), pages(row_bytes=(0, 6)), ikv.IKV_ERR_SHAPE),
    (shape(), cache(), pages(row_bytes=(1, 1 << 28)), ikv.IKV_ERR_SHAPE),
]


@pytest.mark.parametrize("i", range(len(PAGES)))
def test_page_calls_check_their_pool(i):
    s, c, p, want = PAGES[i]
    n = ikv.SZ(0)
    big = ctypes.c_size_t(1 << 30)
    assert status("ikv_pages_workspace_size", s, c, p, ctypes.byref(n)) == want
    assert status("ikv_pages_release", s, c, p, 0, None) == want
    assert status("ikv_pages_fork", s, c, p, 1, A, A, None, None) == want
    assert status("ikv_pages_writable", s, c, p, None, None, 1, None, A, big, None) == want
    assert status("ikv_pages_compact", s, c, p, A, A, None, None, A, big, None) == want


def test_page_calls_check_their_arguments():
    s, c, p, big = shape(), cache(), pages(), ctypes.c_size_t(1 << 30)
    n = ikv.ikv_pages_workspace_size(s, c, p)
    assert n > 0
    assert status("ikv_pages_release", s, c, p, -1, None) == ikv.IKV_ERR_ARG
    assert status("ikv_pages_fork", s, c, p, 3, A, A, None, None) == ikv.IKV_ERR_SHAPE
    assert status("ikv_pages_fork", s, c, p, -1, A, A, None, None) == ikv.IKV_ERR_SHAPE
    assert status("ikv_pages_fork", s, c, p, 1, None, A, None, None) == ikv.IKV_ERR_ARG
    assert status("ikv_pages_writable", s, c, p, None, None, 65, None, A, big, None) == ikv.IKV_ERR_SHAPE
    assert status("ikv_pages_writable", s, c, p, None, None, -1, None, A, big, None) == ikv.IKV_ERR_SHAPE
    for name, args in (("ikv_pages_writable", (None, None, 1, None)), ("ikv_pages_compact", (A, A, None, None))):
        assert status(name, s, c, p, *args, None, big, None) == ikv.IKV_ERR_WORKSPACE
        assert status(name, s, c, p, *args, A, ctypes.c_size_t(n - 1), None) == ikv.IKV_ERR_WORKSPACE
        assert status(name, s, c, p, *args, A + 8, big, None) == ikv.IKV_ERR_ALIGN
    assert status("ikv_pages_compact", s, c, p, None, A, None, None, A, big, None) == ikv.IKV_ERR_ARG


def test_page_calls_refuse_pools_they_cannot_count():
    c, p = cache(num_pages=0x7fffffff), pages()
    assert status("ikv_pages_release", shape(), c, p, 0, None) == ikv.IKV_ERR_SHAPE
    assert status("ikv_pages_workspace_size", shape(), c, p, ctypes.byref(ikv.SZ(0))) == ikv.IKV_ERR_SHAPE


def test_forks_and_compactions_refuse_the_layout_of_per_layer_eviction():
    s, c, p, big = shape(), cache(pos_cap=128), pages(), ctypes.c_size_t(1 << 30)
    assert status("ikv_pages_fork", s, c, p, 1, A, A, A, None) == ikv.IKV_ERR_UNSUPPORTED
    assert status("ikv_pages_compact", s, c, p, A, A, A, None, A, big, None) == ikv.IKV_ERR_UNSUPPORTED


def test_dense_rows_with_strided_channels_are_refused():
    c = Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16)
    x = torch.zeros(1, 2, 8, 2, 64)
    assert c.dense_rows(x.transpose(1, 2)).seq == x.stride(2)
    with pytest.raises(ValueError):
        c.dense_rows(x.transpose(3, 4))


def test_page_calls_do_not_go_by_max_len():
    s, p = shape(), pages()
    n = ikv.ikv_pages_workspace_size(s, cache(), p)
    assert ikv.ikv_pages_workspace_size(s, cache(max_len=1000), p) == n  # a bound past the slot space
    assert status("ikv_pages_release", s, cache(max_len=-1), p, 0, None) == ikv.IKV_ERR_SHAPE
    assert status("ikv_pages_release", s, None, p, 0, None) == ikv.IKV_ERR_ARG
