"""Attention on another stream than the caller's current one, with a workspace that the call makes for itself."""
import pytest
import torch

from test_gpu_shared_prefix import B, Problem  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


def test_a_workspace_made_by_the_call_is_of_the_calls_stream(B):
    """A tensor of the workspace's size is freed while a copy out of it is still queued on the current stream: its memory is that
    stream's to hand out again, so the call on the side stream, which runs at once, must take its workspace elsewhere."""
    p = Problem(B, [30, 2, 55, 9] * 20, 500, 8, 2, 128, 16, seed=40)
    want, want_lse = p.launch()
    size = B.shared_prefix_attention_workspace_bytes(p.cache, p.batch, p.heads)
    assert size > 2 << 20
    q, side = p.q.cuda(), torch.cuda.Stream()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], device="cuda")
    B.shared_prefix_attention_launch(p.cache, p.batch, q, out, lse, softmax_scale=p.scale, stream=side)  # its memory is there from now on
    torch.cuda.synchronize()
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        tensor = torch.full((size,), 7, dtype=torch.uint8, device="cuda")
        copy = torch.empty_like(tensor)
        torch.cuda._sleep(20_000_000)  # about 10 ms of the current stream
        copy.copy_(tensor)
        del tensor
        B.shared_prefix_attention_launch(p.cache, p.batch, q, out, lse, softmax_scale=p.scale, stream=side)
        torch.cuda.synchronize()
        assert bool((copy == 7).all())
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert B.rt_device_status() == 0
