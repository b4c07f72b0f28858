"""Attention over packed prompts where one key outweighs all others and has values of zero: the result comes from small weights alone.

Tolerance: kv_reference.out_tolerance, and for fp16 weights, whose steps do not go below 2^-24, half a step of the factor 2^7 that they
are held with: 2^-32 of the row's largest weight, for every key, times |v| (the denominator is at least that largest weight).  Without the
factor a weight of e^-18 = 2^-26 is less than half a step and counts nothing, one of e^-12 is off by up to 2^-7."""
import math

import pytest
import torch

import kv_reference as R
from test_gpu_prompt import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens", [[(130, 600), (300, 300)], [(20, 3000), (9, 2500)]])  # without parts and with
@pytest.mark.parametrize("gap", [12.0, 15.0, 18.0])
@pytest.mark.parametrize("sink", ["first", "last seen by all"])
def test_small_weights_beside_a_large_one(B, dtype, dim, lens, gap, sink):
    p = Problem(B, lens, 4, 2, dim, dtype, seed=dim + int(gap), fused=False)
    assert (B.prompt_attention_workspace_bytes(p.batch, p.q, p.k) > 0) == (lens[0][1] == 3000)
    g = torch.Generator().manual_seed(1)
    p.q.zero_()
    p.q[..., 0] = math.sqrt(dim)
    p.k[..., 0] = (0.1 * torch.randn(p.k.shape[:2], generator=g)).to(p.dtype).cuda()
    p.v.copy_((500 + 500 * torch.rand(p.v.shape, generator=g)).to(p.dtype))
    for (n_q, n_k), first in zip(lens, p.k_starts):
        at = first + (0 if sink == "first" else n_k - n_q)
        p.k[at, :, 0] = gap
        p.v[at] = 0
    out, lse = p.launch()
    want, want_lse, mean_abs, score_abs, seen, _ = p.reference()
    out, lse = out.double().cpu(), lse.double().cpu()
    tol = R.out_tolerance(want, mean_abs, score_abs, seen, p.dtype, False, dim)
    if dtype == "fp16":
        tol += 2.0 ** -32 * (seen * float(p.v.abs().max())).unsqueeze(-1)
    assert not bool(((out - want).abs() > tol).any()), float(((out - want).abs() / tol).max())
    assert not bool(((lse - want_lse).abs() > R.lse_tolerance(want_lse, score_abs, seen, dim)).any())
    assert B.rt_device_status() == 0
