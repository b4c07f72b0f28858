"""What the binding of the rotary positions refuses before it calls the library, without a GPU."""
import pytest
import torch

from paper_2601_12698_b200 import binding as B


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_tables_and_tensors_off_the_gpu_are_refused(device, monkeypatch):
    """A host address must never reach a launch, not even where table and tensors agree on their device."""
    calls = []
    monkeypatch.setattr(B, "_call_on", lambda *a: calls.append(a) or B.RT_OK)
    monkeypatch.setattr(B, "_stream_of", lambda *a: 0)
    table = B.RotaryTable(64, device="cpu")
    q, positions = torch.zeros(4, 2, 64, device=device), torch.zeros(4, dtype=torch.int64, device=device)
    for kw in ({}, {"k": q[:, :1]}, {"q_out": torch.zeros_like(q)}):
        with pytest.raises(ValueError, match="CUDA device"):
            B.rotary_launch(table, positions, q, **kw)
    assert not calls
    assert table.fractions[0] == B.RotaryTable(64, device="cpu", interleaved=True).fractions[0]  # the frequencies alone need no GPU


@pytest.mark.parametrize("factor,want", [(8.0, 1.2079441541679836), (1.0, 1.0), (0.5, 1.0), (1e-6, 1.0)])
def test_the_ramp_has_a_magnitude_only_where_it_stretches(factor, want):
    """0.1 ln(factor) + 1, which would fall below 1 for factors below 1 and below 0 for those below e^-10."""
    table = B.RotaryTable(64, scaling="yarn", factor=factor, original_len=4096.0, device="cpu")
    assert table.magnitude == pytest.approx(want, rel=2.0 ** -23)
    assert B.RotaryTable(64, scaling="yarn", factor=factor, original_len=4096.0, magnitude=0.75, device="cpu").magnitude == 0.75
