"""Prompts of thousands of tokens, element by element against the 64-bit form (worked out on the GPU): rings and phases of a block turn over
many times within it.  And calls on a stream of their own, with what they read and overwrite ordered before them."""
import pytest
import torch

import prompt_reference as P
from test_gpu_prompt import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


def _reference(p):
    with torch.device("cuda"):
        return tuple(x.cpu() for x in P.attend(p.q, p.k, p.v, p.q_starts, p.k_starts, p.causal, p.scale))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,heads,kv_heads,dim,causal", [
    ([(6000, 6000)], 2, 1, 128, True), ([(5001, 9003)], 2, 2, 64, True), ([(4500, 4500)], 3, 1, 256, True), ([(4099, 5000)], 2, 1, 128, False), ([(5, 5), (4097, 12000), (3001, 40)], 2, 1, 136, True),
    ([(300, 300), (2100, 2100)] * 3, 4, 1, 128, True), ([(1, 70000), (17, 33333)], 4, 1, 256, True)])
def test_long_prompts(B, dtype, lens, heads, kv_heads, dim, causal):
    p = Problem(B, lens, heads, kv_heads, dim, dtype, causal, tail=5, seed=dim)
    first = p.launch()
    p.check(*first, _reference(p))
    for a, b in zip(first, p.launch()):
        assert torch.equal(a, b)
    assert B.rt_device_status() == 0


def test_calls_on_streams_of_their_own(B):
    """With parts and without; the fill of the results is ordered before the call that overwrites it."""
    for lens in ([(30, 4000), (2, 3000)], [(600, 600)]):
        p = Problem(B, lens, 8, 2, 128, seed=6)
        want = p.launch()
        sides = [torch.cuda.Stream() for _ in range(3)]
        outs = [(torch.full_like(want[0], 5.0), torch.full_like(want[1], 5.0)) for _ in sides]
        for side, (out, lse) in zip(sides, outs):
            side.wait_stream(torch.cuda.current_stream())
            B.prompt_attention_launch(p.batch, p.q, p.k, p.v, out, lse, softmax_scale=p.scale, stream=side)
        torch.cuda.synchronize()
        for out, lse in outs:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_pages_copied_on_a_stream_of_their_own(B):
    """The page numbers are written before the stream goes on, and are kept until it is done."""
    cache = B.KvCache.allocate(20, 16, 4, 64, torch.bfloat16)
    for t in (cache.k, cache.v):
        t.copy_(torch.randn(t.shape))
    stack, before = B.KvCacheStack([cache]), [t.clone() for t in (cache.k, cache.v)]
    src, dst = torch.arange(5, dtype=torch.int32, device="cuda") + 3, torch.arange(10, 15, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.kv_cache_copy_pages_launch(stack, src, dst, stream=side)
    side.synchronize()
    for t, old in zip((cache.k, cache.v), before):
        assert torch.equal(t[10:15], old[3:8]) and torch.equal(t[:10], old[:10]) and torch.equal(t[15:], old[15:])
