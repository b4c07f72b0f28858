"""As many layers as a stack holds, bit for bit against indexing."""
import pytest
import torch

from test_gpu_kv_cache import B  # noqa: F401  (a fixture)
from test_gpu_kv_move import _bytes, _check_moves, _compact_reference, _sides, _stack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,fmt", [(64, "int8"), (33, "plain")])
def test_moves_in_all_layers_at_once(B, dim, fmt):
    page, heads = 8, 2
    stack, _ = _stack(B, B.RT_MAX_LAYERS, "token", 24, page, heads, dim, "bf16", fmt)
    g = torch.Generator().manual_seed(dim)
    want = [_bytes(t) for t in _sides(stack)]
    src, dst, tokens = (torch.tensor(x, dtype=torch.int32) for x in ([1, 2, 1], [20, 21, 22], [8, 3, 5]))
    for w in want:
        for s, d, n in zip(src.tolist(), dst.tolist(), tokens.tolist()):
            w[d, :n] = w[s, :n].clone()
    B.kv_cache_copy_pages_launch(stack, src.cuda(), dst.cuda(), tokens.cuda())
    assert all(torch.equal(_bytes(t), w) for t, w in zip(_sides(stack), want))
    table = torch.randperm(18, generator=g).int().reshape(3, 6)
    starts, lens, keep = torch.tensor([4, 0, 9]).int(), torch.tensor([40, -1, 48]).int(), torch.rand(3, 40, generator=g) < 0.5
    new = _compact_reference(want, table, starts, lens, keep, page)
    got = torch.zeros(3, dtype=torch.int32, device="cuda")
    B.kv_cache_compact_launch(stack, table.cuda(), starts.cuda(), lens.cuda(), keep.cuda(), got)
    assert got.tolist() == new
    _check_moves(stack, want, table, lens, new, page)
    assert B.rt_device_status() == 0
