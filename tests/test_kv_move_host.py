"""Refusals of the moves inside a cache, without a GPU (pointers are numbers that nothing follows)."""
import ctypes

import pytest

from paper_2601_12698_b200 import binding as B
from test_kv_cache_host import P, _cache


def _array(*caches):
    return (B.rt_kv_cache * len(caches))(*caches), len(caches)


def _copy(caches=None, src=P, dst=P, tokens=None, n=3):
    return B.lib.kv_cache_copy_pages_launch(*(caches or _array(_cache(), _cache())), src, dst, tokens, n, None)


def _compact(caches=None, table=P, stride=4, width=4, starts=P, lens=P + 64, keep=P, keep_stride=8, window=8, new_lens=P + 128, n=3):
    batch = B.rt_compact_batch(table, starts, lens, keep, new_lens, n, window, stride, width, keep_stride)
    return B.lib.kv_cache_compact_launch(*(caches or _array(_cache(), _cache())), ctypes.byref(batch), None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), "RT_ERR_SHAPE"), (dict(n=(1 << 30) + 1), "RT_ERR_SHAPE"), (dict(src=None), "RT_ERR_NULL"), (dict(dst=None), "RT_ERR_NULL"),
    (dict(src=P + 2), "RT_ERR_ALIGN"), (dict(tokens=P + 1), "RT_ERR_ALIGN")])
def test_copy_refusals(kw, status):
    assert _copy(**kw) == getattr(B, status)
    assert B.lib.rt_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), "RT_ERR_SHAPE"), (dict(n=(1 << 24) + 1), "RT_ERR_SHAPE"), (dict(window=-1), "RT_ERR_SHAPE"), (dict(window=(1 << 30) + 1), "RT_ERR_SHAPE"),
    (dict(width=-1), "RT_ERR_SHAPE"), (dict(width=1 << 31), "RT_ERR_SHAPE"), (dict(stride=-1), "RT_ERR_SHAPE"), (dict(keep_stride=-8), "RT_ERR_SHAPE"), (dict(table=None), "RT_ERR_NULL"),
    (dict(starts=None), "RT_ERR_NULL"), (dict(lens=None), "RT_ERR_NULL"), (dict(keep=None), "RT_ERR_NULL"), (dict(new_lens=None), "RT_ERR_NULL"),
    (dict(table=P + 2), "RT_ERR_ALIGN"), (dict(new_lens=P + 2), "RT_ERR_ALIGN"), (dict(new_lens=P), "RT_ERR_SHAPE"), (dict(new_lens=P + 64), "RT_ERR_SHAPE")])
def test_compact_refusals(kw, status):
    assert _compact(**kw) == getattr(B, status)
    assert B.lib.rt_last_error()


@pytest.mark.parametrize("change", [{"n_pages": 9}, {"page_size": 8}, {"kv_heads": 1}, {"head_dim": 32}, {"format": 1}, {"page_stride": 1 << 12}, {"token_stride": 256},
                                    {"head_stride": 128}, {"scale_page_stride": 64}, {"scale_token_stride": 4}, {"scale_head_stride": 2}])
def test_caches_that_differ_are_refused(change):
    for call in (_copy, _compact):
        assert call(_array(_cache(), _cache(**change))) == B.RT_ERR_SHAPE
        assert call(_array(_cache(k=None))) == B.RT_ERR_NULL
        assert call((None, 2)) == B.RT_ERR_NULL
        assert call((_array(_cache())[0], 0)) == B.RT_ERR_SHAPE
        assert call((_array(_cache())[0], B.RT_MAX_LAYERS + 1)) == B.RT_ERR_SHAPE


def test_nothing_to_do_is_no_error():
    assert _copy(src=None, dst=None, n=0) == B.RT_OK
    assert _compact(table=None, starts=None, lens=None, keep=None, new_lens=None, n=0) == B.RT_OK
    assert B.lib.kv_cache_compact_launch(*_array(_cache()), None, None) == B.RT_ERR_NULL


@pytest.mark.parametrize("at", [P + 4, P - 8, P + 60, P + 72, P + 56])
def test_new_lengths_that_overlap_the_inputs_are_refused(at):
    assert _compact(new_lens=at) == B.RT_ERR_SHAPE and "overlap" in B.lib.rt_last_error().decode()


def test_pages_that_are_too_large_are_refused():
    wide = dict(page_size=1 << 16, kv_heads=256, head_dim=128, head_stride=128, token_stride=256 * 128, page_stride=256 * 128 << 16)
    assert _copy(_array(_cache(**wide))) == B.RT_ERR_SHAPE and B.lib.rt_last_error()
