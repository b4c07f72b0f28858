"""What the binding of the attention does around the library's call, with stand-ins for the library and the device."""
import contextlib
import types

import pytest
import torch

from paper_2601_12698_b200 import binding as B


@pytest.fixture
def device(monkeypatch):
    """CPU tensors name the device -1, and so does this stand-in; it notes which stream is current at each step."""
    seen = types.SimpleNamespace(current="caller's", events=[])

    @contextlib.contextmanager
    def on(stream):
        before = seen.current
        seen.current = before if stream is None else stream.name
        yield
        seen.current = before

    def workspace(cache, batch, q_heads):
        seen.events.append(("allocate", seen.current))
        return torch.empty(64, dtype=torch.uint8)

    def launch(*args):
        seen.events.append(("launch", args[-1]))
        return 0

    core = types.SimpleNamespace(_cuda_getDevice=lambda: -1, _cuda_getCurrentRawStream=lambda index: 11)
    monkeypatch.setattr(B, "_torch", types.SimpleNamespace(float32=torch.float32, cuda=types.SimpleNamespace(stream=on), _C=core))
    monkeypatch.setattr(B, "_TORCH_CODES", {torch.bfloat16: B.RT_BF16})
    monkeypatch.setattr(B, "lib", types.SimpleNamespace(shared_prefix_attention_launch=launch))
    monkeypatch.setattr(B, "shared_prefix_attention_workspace", workspace)
    return seen


def _call(**kw):
    cache = types.SimpleNamespace(head_dim=64, device_index=-1, _ref=None)
    batch = types.SimpleNamespace(n_seqs=2, q_len=1, device_index=-1, _ref=None)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    B.shared_prefix_attention_launch(cache, batch, q, torch.zeros_like(q), **kw)


def test_a_workspace_made_by_the_call_belongs_to_the_stream_that_uses_it(device):
    """Memory that the caller's stream may still be using is free for that stream's next use only: a workspace for another stream has
    to come from that stream's own."""
    _call(stream=types.SimpleNamespace(name="side", device_index=-1, cuda_stream=22))
    assert device.events == [("allocate", "side"), ("launch", 22)]
    device.events.clear()
    _call()
    assert device.events == [("allocate", "caller's"), ("launch", 11)]
    device.events.clear()
    _call(stream=types.SimpleNamespace(name="side", device_index=-1, cuda_stream=22), workspace=torch.empty(64, dtype=torch.uint8))
    assert device.events == [("launch", 22)]


def test_a_stream_of_another_device_is_refused_before_anything_is_made(device):
    with pytest.raises(ValueError):
        _call(stream=types.SimpleNamespace(name="side", device_index=1, cuda_stream=22))
    assert device.events == []
