"""Refusals of the cache's and the shared-prefix attention's C entry points: argument errors are reported before any device is
asked for, so these run without a GPU (pointers are numbers that nothing dereferences)."""
import ctypes

import pytest

from paper_2601_12698_b200 import binding as B

P = 1 << 20  # a pointer that is never followed


def _cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=8, page_size=16, kv_heads=2, head_dim=64, format=B.RT_KV_INT8, dtype=0, reserved=0,
             page_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64, scale_page_stride=32, scale_token_stride=2, scale_head_stride=1)
    d.update(kw)
    return B.rt_kv_cache(**d)


def _batch(**kw):
    d = dict(prefix_pages=P, page_table=P, suffix_lens=P, prefix_len=100, max_suffix_len=30, n_seqs=3, page_table_stride=2,
             page_table_width=2, n_prefix_pages=7, q_len=1, reserved=0)
    d.update(kw)
    return B.rt_prefix_batch(**d)


@pytest.mark.parametrize("change,status", [
    ({"format": 3}, "RT_ERR_DTYPE"), ({"format": -1}, "RT_ERR_DTYPE"), ({"format": 0, "dtype": 5}, "RT_ERR_DTYPE"),
    ({"format": 0, "dtype": 1}, "RT_ERR_DTYPE"), ({"page_size": 0}, "RT_ERR_SHAPE"), ({"page_size": 65537}, "RT_ERR_SHAPE"),
    ({"kv_heads": 0}, "RT_ERR_SHAPE"), ({"head_dim": 0}, "RT_ERR_SHAPE"), ({"head_dim": 257}, "RT_ERR_SHAPE"), ({"n_pages": -1}, "RT_ERR_SHAPE"),
    ({"token_stride": -1}, "RT_ERR_SHAPE"), ({"scale_head_stride": -4}, "RT_ERR_SHAPE"), ({"k": None}, "RT_ERR_NULL"), ({"v_scale": None}, "RT_ERR_NULL"),
    ({"k_scale": P + 2}, "RT_ERR_ALIGN"), ({"format": 0, "k": P + 1}, "RT_ERR_ALIGN")])
def test_cache_refusals(change, status):
    c = _cache(**change)
    want = getattr(B, status)
    assert B.lib.kv_cache_write_launch(ctypes.byref(c), P, 128, 64, P, 128, 64, P, 5, 0, None) == want
    assert B.lib.kv_cache_read_launch(ctypes.byref(c), P, 5, P, 128, 64, P, 128, 64, 0, None) == want
    assert B.lib.rt_last_error()


def test_cache_call_refusals():
    c = ctypes.byref(_cache())
    call = B.lib.kv_cache_write_launch
    assert call(None, P, 128, 64, P, 128, 64, P, 5, 0, None) == B.RT_ERR_NULL
    assert call(c, None, 128, 64, P, 128, 64, P, 5, 0, None) == B.RT_ERR_NULL
    assert call(c, P, 128, 64, P, 128, 64, None, 5, 0, None) == B.RT_ERR_NULL
    assert call(c, P, 128, 64, P, 128, 64, P, -1, 0, None) == B.RT_ERR_SHAPE
    assert call(c, P, -128, 64, P, 128, 64, P, 5, 0, None) == B.RT_ERR_SHAPE
    assert call(c, P, 128, 64, P, 128, 64, P, 5, 3, None) == B.RT_ERR_DTYPE
    assert call(c, P + 1, 128, 64, P, 128, 64, P, 5, 0, None) == B.RT_ERR_ALIGN
    assert call(c, P, 128, 64, P, 128, 64, P + 4, 5, 0, None) == B.RT_ERR_ALIGN
    assert call(c, None, 0, 0, None, 0, 0, None, 0, 0, None) == B.RT_OK  # no tokens: nothing is needed


@pytest.mark.parametrize("cache,batch,heads,status", [
    ({}, {"q_len": 0}, 4, "RT_ERR_SHAPE"), ({}, {"q_len": 17}, 4, "RT_ERR_SHAPE"), ({}, {}, 3, "RT_ERR_SHAPE"), ({}, {}, 0, "RT_ERR_SHAPE"),
    ({"head_dim": 72}, {}, 4, "RT_ERR_SHAPE"), ({"head_dim": 60, "format": 0}, {}, 4, "RT_ERR_SHAPE"), ({}, {"prefix_len": 113}, 4, "RT_ERR_SHAPE"),
    ({}, {"max_suffix_len": 33}, 4, "RT_ERR_SHAPE"), ({}, {"n_seqs": -1}, 4, "RT_ERR_SHAPE"), ({}, {"n_seqs": 1 << 30}, 4, "RT_ERR_SHAPE"),
    ({}, {"prefix_len": (1 << 30) + 1, "n_prefix_pages": 1 << 30}, 4, "RT_ERR_SHAPE"), ({"page_size": 0}, {}, 4, "RT_ERR_SHAPE"), ({"format": 9}, {}, 4, "RT_ERR_DTYPE")])
def test_attention_geometry_refusals(cache, batch, heads, status):
    c, b = _cache(**cache), _batch(**batch)
    got = B.lib.shared_prefix_attention_launch(ctypes.byref(c), ctypes.byref(b), P, heads * 64, 64, heads, P, P, 0.125, 0, P, 1 << 40, None)
    assert got == getattr(B, status)
    assert B.lib.shared_prefix_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), heads) == -1
    assert B.lib.rt_last_error()


def test_attention_null_batch_and_type():
    c, b = _cache(), _batch()
    call = B.lib.shared_prefix_attention_launch
    assert call(ctypes.byref(c), None, P, 256, 64, 4, P, P, 0.125, 0, P, 1 << 40, None) == B.RT_ERR_NULL
    assert call(None, ctypes.byref(b), P, 256, 64, 4, P, P, 0.125, 0, P, 1 << 40, None) == B.RT_ERR_NULL
    assert call(ctypes.byref(c), ctypes.byref(b), P, 256, 64, 4, P, P, 0.125, B.RT_FP32, P, 1 << 40, None) == B.RT_ERR_DTYPE


def test_struct_layouts_match_the_header():
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {"rt_kv_cache": B.rt_kv_cache, "rt_prefix_batch": B.rt_prefix_batch}
    lines = [f'printf("%zu\\n", sizeof({n}));' + "".join(f'printf("%zu\\n", offsetof({n}, {f}));' for f, _ in t._fields_) for n, t in fields.items()]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "rmsnorm_tuner.h"\nint main(void){' + "".join(lines) + "return 0;}\n"
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "s.c"), "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "s")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for t in fields.values():
        want += [ctypes.sizeof(t)] + [getattr(t, f).offset for f, _ in t._fields_]
    assert got == want
    assert (B.RT_ERR_INDEX, B.RT_KV_MAX_HEAD_DIM, B.RT_MAX_QUERY_LEN) == (12, 256, 16)
