"""What the shared-prefix and the sliding-window calls refuse, on the host, before any launch."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_03515_gb300 import ikv

    return ikv


BIG = 1 << 44


def _shape(lib, **kw):
    d = dict(batch=2, layers=2, q_heads=8, kv_heads=2, head_dim=128, dtype=lib.IKV_BF16, granularity=lib.IKV_GRAN_SEQ)
    d.update(kw)
    return lib.ikv_shape(**d)


def _cache(lib, **kw):
    d = dict(k=16, v=16, block_table=16, num_pages=4, page_size=64, max_pages=4, len=16, pos=16, next_pos=16, max_len=100)
    d.update(kw)
    return lib.ikv_cache(**d)


def _window(lib, shape=None, cache=None, layer=0, q=16, out=16, ws=16, ws_bytes=BIG, **kw):
    d = dict(window=100, sinks=4, row0=None, count=None, max_count=3, q_stride=0, out_stride=0)
    d.update(kw)
    return lib.raw_status("ikv_window_attend", shape or _shape(lib), cache or _cache(lib), lib.ikv_window(**d), layer, q,
                          out, ws, ws_bytes, None)


def _prefix(lib, shape=None, cache=None, layer=0, q=16, out=16, score=None, ema=None, alpha=0.5, ws=16, ws_bytes=BIG, **kw):
    d = dict(n_groups=1, first=16, member=16, len=16)
    d.update(kw)
    return lib.raw_status("ikv_prefix_attend_score", shape or _shape(lib), cache or _cache(lib), lib.ikv_prefix(**d), layer,
                          q, out, score, ema, alpha, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_window, _prefix])
def test_shapes_caches_and_pointers(lib, call):
    for kw, want in [
        (dict(shape=_shape(lib, head_dim=96)), lib.IKV_ERR_UNSUPPORTED),
        (dict(shape=_shape(lib, q_heads=6)), lib.IKV_ERR_UNSUPPORTED),
        (dict(shape=_shape(lib, q_heads=9)), lib.IKV_ERR_SHAPE),
        (dict(shape=_shape(lib, batch=0)), lib.IKV_ERR_SHAPE),
        (dict(shape=_shape(lib, q_heads=16384, kv_heads=16384)), lib.IKV_ERR_SHAPE),
        (dict(shape=_shape(lib, dtype=5)), lib.IKV_ERR_ARG),
        (dict(cache=_cache(lib, k=0)), lib.IKV_ERR_ARG),
        (dict(cache=_cache(lib, v=8)), lib.IKV_ERR_ALIGN),
        (dict(cache=_cache(lib, page_size=0)), lib.IKV_ERR_SHAPE),
        (dict(cache=_cache(lib, code_bits=4)), lib.IKV_ERR_UNSUPPORTED),
        (dict(cache=_cache(lib, dead_slots=1, pos=0)), lib.IKV_ERR_ARG),
        (dict(layer=2), lib.IKV_ERR_ARG),
        (dict(layer=-1), lib.IKV_ERR_ARG),
        (dict(q=None), lib.IKV_ERR_ARG),
        (dict(out=None), lib.IKV_ERR_ARG),
        (dict(q=8), lib.IKV_ERR_ALIGN),
        (dict(out=24), lib.IKV_ERR_ALIGN),
        (dict(ws=None), lib.IKV_ERR_WORKSPACE),
        (dict(ws_bytes=1000), lib.IKV_ERR_WORKSPACE),
        (dict(ws=8), lib.IKV_ERR_ALIGN),
    ]:
        assert call(lib, **kw) == want, (kw, lib.ikv_last_error())
        assert lib.ikv_last_error() != ""


def test_window_arguments(lib):
    for kw, want in [
        (dict(window=-1), lib.IKV_ERR_ARG),
        (dict(sinks=-1), lib.IKV_ERR_ARG),
        (dict(max_count=-1), lib.IKV_ERR_ARG),
        (dict(max_count=1 << 27), lib.IKV_ERR_SHAPE),
        (dict(max_count=2**31 - 1), lib.IKV_ERR_SHAPE),
        (dict(q_stride=1016), lib.IKV_ERR_SHAPE),
        (dict(out_stride=-1024), lib.IKV_ERR_SHAPE),
        (dict(q_stride=1028), lib.IKV_ERR_ALIGN),
        (dict(out_stride=1025), lib.IKV_ERR_ALIGN),
    ]:
        assert _window(lib, **kw) == want, (kw, lib.ikv_last_error())
    # more work than a CTA's share can be counted for
    huge = _cache(lib, page_size=64, max_pages=1 << 23)
    assert _window(lib, cache=huge, shape=_shape(lib, batch=64), max_count=4096) == lib.IKV_ERR_SHAPE
    assert _prefix(lib, cache=huge, shape=_shape(lib, batch=1 << 20)) == lib.IKV_ERR_SHAPE
    n = lib.SZ(0)
    w = lib.ikv_window(0, 0, None, None, 1, 0, 0)
    assert lib.raw_status("ikv_window_workspace_size", _shape(lib), _cache(lib), None, ctypes.byref(n)) == lib.IKV_ERR_ARG
    assert lib.raw_status("ikv_window_workspace_size", _shape(lib), _cache(lib), w, None) == lib.IKV_ERR_ARG
    assert lib.raw_status("ikv_window_workspace_size", _shape(lib), _cache(lib), w, ctypes.byref(n)) == lib.IKV_OK
    assert n.value > 0
    # nothing to do: no query
    assert _window(lib, max_count=0) == lib.IKV_OK


def test_prefix_arguments(lib):
    for kw, want in [
        (dict(n_groups=-1), lib.IKV_ERR_ARG),
        (dict(first=None), lib.IKV_ERR_ARG),
        (dict(member=None), lib.IKV_ERR_ARG),
        (dict(len=None), lib.IKV_ERR_ARG),
        (dict(n_groups=1 << 21), lib.IKV_ERR_SHAPE),
        (dict(ema=16, alpha=1.5), lib.IKV_ERR_ARG),
        (dict(ema=16, alpha=float("nan")), lib.IKV_ERR_ARG),
        (dict(shape=_shape(lib, batch=1 << 26)), lib.IKV_ERR_SHAPE),
    ]:
        assert _prefix(lib, **kw) == want, (kw, lib.ikv_last_error())
    n = lib.SZ(0)
    p = lib.ikv_prefix(0, None, None, None)
    assert lib.raw_status("ikv_prefix_workspace_size", _shape(lib), _cache(lib), None, ctypes.byref(n)) == lib.IKV_ERR_ARG
    assert lib.raw_status("ikv_prefix_workspace_size", _shape(lib), _cache(lib), p, None) == lib.IKV_ERR_ARG
    assert lib.raw_status("ikv_prefix_workspace_size", _shape(lib), _cache(lib), p, ctypes.byref(n)) == lib.IKV_OK
    assert n.value > 0
