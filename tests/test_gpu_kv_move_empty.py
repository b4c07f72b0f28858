"""Moves in caches without a page."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("layers", [1, 3])
def test_caches_without_pages_can_be_stacked(B, dtype, layers):
    stack = B.KvCacheStack([B.KvCache.allocate(0, 16, 2, 64, dtype) for _ in range(layers)])
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    B.rt_device_status()
    B.kv_cache_copy_pages_launch(stack, i32(-1, 0), i32(0, -1))
    B.kv_cache_copy_pages_launch(stack, i32(), i32())
    table, keep, new = torch.empty(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, 8, dtype=torch.bool, device="cuda"), i32(9, 9, 9)
    B.kv_cache_compact_launch(stack, table, i32(0, 0, 0), i32(0, -1, 0), keep, new)
    assert new.tolist() == [0, -1, 0] and B.rt_device_status() == 0
    B.kv_cache_copy_pages_launch(stack, i32(0), i32(1))
    assert B.rt_device_status() == B.RT_ERR_INDEX
    B.kv_cache_compact_launch(stack, i32(0, 0, 0)[:, None], i32(0, 0, 0), i32(8, 8, 0), keep.logical_not(), new)
    assert new.tolist() == [8, 8, 0] and B.rt_device_status() == 0  # all of them stay where they are
    keep[:, 1] = True
    B.kv_cache_compact_launch(stack, i32(0, 0, 0)[:, None], i32(0, 0, 0), i32(8, -1, 0), keep, new)
    assert new.tolist() == [1, -1, 0] and B.rt_device_status() == B.RT_ERR_INDEX
