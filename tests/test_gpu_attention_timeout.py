"""Waits of the attention kernels that run out on purpose, in the way that harms nothing (see test_gpu_timeout.py): tiles are fetched
but never announced (keys first), or their places never published (tiles form), and the poll limit is low.  The launch goes through all
its barriers, reports the status, and the next call with waits as usual is right."""
import pytest
import torch

from test_gpu_prefix_alone import reference
from test_gpu_shared_prefix import B, Problem  # noqa: F401  (B is a fixture)
from test_gpu_timeout import _expiring_waits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["plain", "e4m3"])
@pytest.mark.parametrize("lens,prefix,heads,kv_heads,dim,q_len", [
    ([300, 20, -1], 0, 4, 1, 128, 2),          # suffixes, 16 rows to a CTA
    ([300, 20], 700, 4, 1, 64, 1),             # prefix and suffixes in one launch
    ([300, 20, 90], 200, 64, 1, 256, 1),       # heads of 256, 64 rows to a CTA
    ([0] * 40, 1500, 8, 2, 128, 1),            # the tiles form, wide
    ([40, 200] * 40, 1500, 1, 1, 64, 1),       # the tiles form, narrow, with suffixes beside it
])
def test_an_expired_wait_is_reported_and_the_next_call_is_right(B, fmt, lens, prefix, heads, kv_heads, dim, q_len):
    p = Problem(B, lens, prefix, heads, kv_heads, dim, 16, "bf16", fmt, q_len, seed=len(lens))
    ref = reference(p)
    p.check(*p.launch(), ref)
    with _expiring_waits(B, polls=50):
        out, lse = p.launch()
        assert out.shape == p.q.shape and lse.shape == p.q.shape[:-1]
        assert B.rt_device_status() == B.RT_ERR_DEVICE_TIMEOUT  # after the launch has completed: it synchronises
        assert B.rt_device_status() == 0
    for _ in range(2):
        p.check(*p.launch(), ref)
