"""The plan of the attention over packed prompts, without a GPU: the entry point is compiled with stand-ins for the device
(prompt_plan_host.cu), 148 SMs."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2601_12698_b200 import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
P = 1 << 20  # an address that nothing follows
MOST = (1 << 63) - 1


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    path = str(tmp_path_factory.mktemp("plan") / "plan.so")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-o", path, os.path.join(HERE, "prompt_plan_host.cu")], check=True)
    lib = ctypes.CDLL(path)
    lib.harness_more_waits.argtypes = [ctypes.c_int64] * 2
    return lib


@pytest.fixture(scope="module")
def workspace(harness):
    fn = harness.prompt_attention_workspace_bytes
    fn.argtypes, fn.restype = B.lib.prompt_attention_workspace_bytes.argtypes, ctypes.c_int64
    return lambda seqs, q, k, max_q, max_k, heads=8, kv_heads=2, dim=128: fn(
        ctypes.byref(B.rt_prompt_batch(P, P, seqs, q, k, max_q, max_k, 1, 0)), heads, kv_heads, dim)


def test_few_queries_behind_many_keys_are_cut_into_parts(workspace):
    assert workspace(1, 40, 3000, 40, 3000) > 0
    assert workspace(1, 40, 500, 40, 500) == 0


@pytest.mark.parametrize("seqs,q,k", [(1, 40, 3000), (3, 45, 5100), (1, 1, 100000), (2, 300, 20000), (1, 0, 0), (1 << 24, 1 << 30, 1 << 30), (1, 1 << 30, 1 << 30)])
@pytest.mark.parametrize("dim", [64, 256])
def test_lengths_beyond_the_tensors_say_no_more_than_these(workspace, seqs, q, k, dim):
    want = workspace(seqs, q, k, q, k, dim=dim)
    assert want >= 0
    for max_q, max_k in ((MOST, MOST), (q, MOST), (MOST, k), (MOST - 127, MOST - 63), (1 << 62, 1 << 40)):
        assert workspace(seqs, q, k, max_q, max_k, dim=dim) == want


def test_the_workspace_holds_every_part(workspace):
    """Results and logarithms of all rows, binary32, for each part, and the flag; parts are never more than 32."""
    for q, k in ((1, 30000), (100, 30000), (512, 16512), (2000, 9000)):
        for dim in (64, 128, 256):
            size, rows = workspace(1, q, k, q, k, 32, 8, dim), q * 32
            if size:
                parts = size // (rows * (dim * 4 + 4))
                assert 2 <= parts <= 32 and parts * rows * (dim * 4 + 4) + 4 <= size < parts * rows * (dim * 4 + 4) + 4 + 16


@pytest.mark.parametrize("keys", [0, 1000, 1 << 20, 15 << 20, 1 << 27, 1 << 30])
@pytest.mark.parametrize("seqs", [1, 1000, 1 << 20, 1 << 24])
def test_a_wait_for_an_item_outlasts_it(harness, keys, seqs):
    """Cycles: a key tile of an item takes up to 6000, and two items may have to pass; 32 sequences take about 800 to go through, once for each of
    up to 31 powers of two of the blocks' costs and once to count."""
    second = 2_000_000_000
    most = -(-keys // 128) * 12000 + -(-seqs // 32) * 800 * 32
    more = harness.harness_more_waits(keys, seqs)
    assert (more + 1) * second >= most and (more <= 80)
    if keys <= 15_000_000 and seqs <= 100_000:
        assert more == 0  # what hangs is found within a second
