"""The plan of the attention over a shared prefix and the arguments of its launches, without a GPU: the entry point is compiled
with stand-ins for the device (attention_plan_host.cu), 148 SMs unless a test says otherwise."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from paper_2601_12698_b200 import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
TILES, KEYS16, KEYS64, MERGE = range(4)
P, WORKSPACE = 1 << 20, 1 << 30  # addresses that nothing follows


class Launch(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("threads", ctypes.c_int32), ("ctas", ctypes.c_int64), ("prefix_parts", ctypes.c_int32),
                ("suffix_parts", ctypes.c_int32), ("prefix_ctas", ctypes.c_int32), ("run", ctypes.c_int32), ("part_out", ctypes.c_int64),
                ("part_lse", ctypes.c_int64)]


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    path = str(tmp_path_factory.mktemp("plan") / "plan.so")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-o", path, os.path.join(HERE, "attention_plan_host.cu")], check=True)
    lib = ctypes.CDLL(path)
    lib.shared_prefix_attention_launch.argtypes = B.lib.shared_prefix_attention_launch.argtypes
    lib.shared_prefix_attention_workspace_bytes.argtypes = B.lib.shared_prefix_attention_workspace_bytes.argtypes
    lib.shared_prefix_attention_workspace_bytes.restype = ctypes.c_int64
    return lib


def _structs(seqs, prefix, suffix, kv_heads, dim, q_len, fmt, page):
    cache = B.rt_kv_cache(P, P, P, P, 1 << 20, page, kv_heads, dim, fmt, B.RT_BF16, 0, page * kv_heads * dim, kv_heads * dim, dim,
                          page * kv_heads, kv_heads, 1)
    width = -(-suffix // page)
    batch = B.rt_prefix_batch(P if prefix else None, P if suffix else None, P, prefix, suffix, seqs, width, width, -(-prefix // page), q_len, 0)
    return cache, batch


def _plan(lib, seqs, prefix, suffix, heads, kv_heads, dim, q_len=1, fmt=B.RT_KV_PLAIN, page=16, sm_count=148):
    """(bytes of workspace, the launches) of one call."""
    cache, batch = _structs(seqs, prefix, suffix, kv_heads, dim, q_len, fmt, page)
    lib.harness_reset(sm_count)
    size = lib.shared_prefix_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), heads)
    assert size >= 0
    status = lib.shared_prefix_attention_launch(ctypes.byref(cache), ctypes.byref(batch), P, heads * dim, dim, heads, P, P, 0.1, B.RT_BF16,
                                                WORKSPACE if size else None, size, None)
    assert status == B.RT_OK
    out = (Launch * 8)()
    return size, [out[i] for i in range(lib.harness_launches(out))]


def _check(seqs, dim, heads, q_len, size, launches):
    """Every launch that leaves parts has a place for them inside the workspace, and what was left in parts is joined."""
    kinds = [l.kernel for l in launches]
    rows = seqs * q_len * heads
    joined = kinds[-1] == MERGE
    assert kinds.count(MERGE) == int(joined)
    for l in launches:
        parts = l.prefix_parts + l.suffix_parts
        if l.kernel == TILES:
            assert joined, "the tiles kernel leaves parts, which nothing joins"
        if joined and parts > 0:
            end_out, end_lse = l.part_out + parts * rows * dim * 4, l.part_lse + parts * rows * 4
            assert l.part_out == WORKSPACE and l.part_lse >= end_out and end_lse <= WORKSPACE + size
            assert l.part_out % 16 == 0 and l.part_lse % 4 == 0
        if not joined:
            assert kinds == [l.kernel] and l.kernel in (KEYS16, KEYS64) and parts == 1 and size == 0
    assert 0 < len(launches) <= 3


@pytest.mark.parametrize("seqs,prefix,heads,kv_heads,dim,q_len", [
    (40, 128, 32, 8, 128, 1), (64, 100, 32, 8, 128, 1), (256, 128, 32, 8, 128, 1), (128, 1, 32, 8, 64, 1), (1024, 5000, 32, 8, 128, 1),
    (512, 4096, 64, 8, 128, 1), (2048, 4096, 32, 32, 64, 1), (65, 128, 1, 1, 64, 1), (16, 128, 8, 1, 128, 1), (75, 100, 4, 1, 64, 1), (20, 90, 16, 1, 96, 8)])
def test_a_prefix_alone_has_a_place_for_its_part(harness, seqs, prefix, heads, kv_heads, dim, q_len):
    for fmt in (B.RT_KV_PLAIN, B.RT_KV_E4M3, B.RT_KV_INT8):
        size, launches = _plan(harness, seqs, prefix, 0, heads, kv_heads, dim, q_len, fmt)
        assert [l.kernel for l in launches] == [TILES, MERGE]
        assert size >= seqs * q_len * heads * (dim + 1) * 4
        _check(seqs, dim, heads, q_len, size, launches)


def test_parts_of_any_geometry_lie_inside_the_workspace(harness):
    rng = random.Random(1)
    wave = lambda hi: int(2 ** rng.uniform(0, hi))
    for _ in range(4000):
        kv_heads, q_len, dim = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 1, 2, 5, 16]), rng.choice([16, 64, 80, 128, 144, 256])
        heads, seqs = kv_heads * rng.choice([1, 2, 4, 5, 16]), wave(11)
        prefix, suffix = rng.choice([0, wave(7), wave(16)]), rng.choice([0, wave(7), wave(15)])
        size, launches = _plan(harness, seqs, prefix, suffix, heads, kv_heads, dim, q_len, rng.choice([0, 1, 2]), rng.choice([1, 16, 24, 128]),
                               rng.choice([148, 148, 132, 1]))
        _check(seqs, dim, heads, q_len, size, launches)


def test_a_workspace_that_is_missing_or_too_small_is_refused(harness):
    for seqs, prefix, suffix in ((40, 128, 0), (256, 32768, 0), (40, 128, 100), (2, 512, 64), (1, 0, 5000)):
        cache, batch = _structs(seqs, prefix, suffix, 8, 128, 1, B.RT_KV_PLAIN, 16)
        harness.harness_reset(148)
        size = harness.shared_prefix_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), 32)
        call = lambda at, n: harness.shared_prefix_attention_launch(ctypes.byref(cache), ctypes.byref(batch), P, 32 * 128, 128, 32, P, P, 0.1,
                                                                    B.RT_BF16, at, n, None)
        assert size > 0
        assert call(None, 0) == B.RT_ERR_NULL and call(WORKSPACE, 0) == B.RT_ERR_CAPACITY and call(WORKSPACE, size - 1) == B.RT_ERR_CAPACITY
        assert call(WORKSPACE + 4, size) == B.RT_ERR_ALIGN
        assert harness.harness_launches((Launch * 8)()) == 0
        assert call(WORKSPACE, size) == B.RT_OK
