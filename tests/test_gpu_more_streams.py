"""The newer serving operators on other streams and in graphs that share nothing but the inputs, past 32 bits of offset, and with heads, tokens or
pages that are not there."""
import pytest
import torch

import prompt_reference as P
from test_gpu_prompt import B, Problem  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


def test_two_captured_calls_side_by_side(B):
    p = Problem(B, [(20, 3000), (100, 100)], 8, 2, 128, seed=3)
    want = p.launch()
    sides, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    torch.cuda.synchronize()
    for _ in range(2):
        out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
        space = B.prompt_attention_workspace(p.batch, p.q, p.k)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(3):
                B.prompt_attention_launch(p.batch, p.q, p.k, p.v, out, lse, space, softmax_scale=p.scale)
        graphs.append(graph)
        outs.append((out, lse, space))
    for _ in range(3):
        for s, g in zip(sides, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for out, lse, _ in outs:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_attention_behind_rows_past_32_bits(B):
    """Queries, keys and values whose last rows lie more than 2^31 elements behind the first."""
    rows, heads, dim = (1 << 31) // (8 * 128) + 300, 8, 128
    q = torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda")
    n, g = 200, torch.Generator().manual_seed(0)
    tail = torch.randn(n, heads, dim, generator=g).to(torch.bfloat16)
    q[rows - n:] = tail.cuda()
    k = v = q[:, :2]
    starts = torch.tensor([rows - n, rows - 50, rows], dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 5.0), torch.full((rows, heads), 5.0, device="cuda")
    B.prompt_attention_launch(B.PromptBatch(starts, n), q, k, v, out, lse)
    want = P.attend(tail, tail[:, :2], tail[:, :2], [0, n - 50, n], [0, n - 50, n], True, dim ** -0.5)
    import kv_reference as R
    tol = R.out_tolerance(want[0], want[2], want[3], want[4], torch.bfloat16, False, dim)
    assert not bool(((out[rows - n:].double().cpu() - want[0]).abs() > tol).any())
    assert bool((out[:rows - n] == 5.0).all()) and bool((lse[:rows - n] == 5.0).all())
    assert B.rt_device_status() == 0


def test_rotary_and_pages_past_32_bits(B):
    rows = (1 << 31) // (8 * 128) + 64
    q = torch.zeros(rows, 8, 128, dtype=torch.bfloat16, device="cuda")
    q[-64:] = torch.randn(64, 8, 128, device="cuda").to(torch.bfloat16)
    positions = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    positions[-64:] = torch.arange(64, device="cuda")
    table, want = B.RotaryTable(128), q[-64:].clone()
    B.rotary_launch(table, positions[-64:].contiguous(), want)
    B.rotary_launch(table, positions, q)
    assert torch.equal(q[-64:], want) and not bool(q[:-64].any())
    cache = B.KvCache(q.view(-1, 16, 8, 128), q.view(-1, 16, 8, 128).clone())
    last = cache.n_pages - 1
    src, dst = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (last, 0))
    B.kv_cache_copy_pages_launch(B.KvCacheStack([cache]), src, dst)
    assert torch.equal(cache.k[0], cache.k[last]) and torch.equal(cache.v[0], cache.v[last])
    pages = torch.tensor([[last - 1, last]], dtype=torch.int32, device="cuda")
    moved = cache.k[last, 8:].clone()
    keep, new = torch.zeros(1, 32, dtype=torch.bool, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    keep[0, 24:] = True
    zero, full = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), 32, dtype=torch.int32, device="cuda")
    B.kv_cache_compact_launch(B.KvCacheStack([cache]), pages, zero, full, keep, new)
    assert new.item() == 8 and torch.equal(cache.k[last - 1, :8], moved)
    assert B.rt_device_status() == 0


def test_nothing_there(B):
    q = torch.randn(10, 4, 64, device="cuda").to(torch.bfloat16)
    k = q[:, :2]
    out, lse = torch.full_like(q, 5.0), torch.full((10, 4), 5.0, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.prompt_attention_launch(B.PromptBatch(one, 0), q, k, k, out, lse)                       # no sequences
    assert bool((out == 5.0).all())
    two = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.prompt_attention_launch(B.PromptBatch(two, 10, none, 0), q, k[:0], k[:0], out, lse)     # no keys at all
    assert bool((out == 0).all()) and bool(torch.isinf(lse).all())
    B.prompt_attention_launch(B.PromptBatch(two, 10), q[:0], k, k, out[:0], lse[:0])          # no rows
    cache = B.KvCache.allocate(4, 16, 2, 64, torch.int8)
    stack = B.KvCacheStack([cache])
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    B.kv_cache_copy_pages_launch(stack, empty, empty)
    B.kv_cache_compact_launch(stack, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), empty, empty, torch.zeros(0, 4, dtype=torch.bool, device="cuda"), empty.clone())
    lens, new = torch.tensor([5], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.kv_cache_compact_launch(stack, torch.zeros(1, 3, dtype=torch.int32, device="cuda"), lens, lens.clone(), torch.zeros(1, 0, dtype=torch.bool, device="cuda"), new)
    assert new.item() == 5 and B.rt_device_status() == 0
