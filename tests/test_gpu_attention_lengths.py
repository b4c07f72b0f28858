"""Suffix lengths beyond the declared bound, where the bound is zero and nothing reads the suffixes."""
import pytest
import torch

from test_gpu_prefix_alone import reference
from test_gpu_shared_prefix import B, Problem  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,prefix,heads,kv_heads,dim", [
    (3, 40, 8, 2, 128),      # few rows, one part
    (3, 5000, 8, 8, 64),     # few rows, joined parts
    (40, 128, 32, 8, 128),   # the tiles form
    (3, 0, 8, 2, 64),        # nothing to see
])
def test_lengths_beyond_a_bound_of_zero_are_cut_and_reported(B, seqs, prefix, heads, kv_heads, dim):
    p = Problem(B, [0] * (seqs - 1) + [-1], prefix, heads, kv_heads, dim, 16, seed=seqs)
    ref = reference(p)
    assert B.rt_device_status() == 0
    out, lse = p.launch()
    p.check(out, lse, ref)
    p.dev_lens[1] = 5
    out, lse = p.launch()
    assert B.rt_device_status() == B.RT_ERR_INDEX and B.rt_device_status() == 0
    p.check(out, lse, ref)
