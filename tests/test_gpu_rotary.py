"""Rotary positions against the plain 64-bit form, element by element.

Tolerance.  A cosine or sine is off by the angle's rounding (the place on the circle to 2^-33 turns, its conversion to binary32
2^-25 of up to half a turn: 1.0e-7 in all), by the function's own unit in the last place (2^-23) and by the product with
the magnitude (2^-24): below 2^-21 of the magnitude.  Two products, a sum: 2^-23 of |x1| + |x2| more.  Then one rounding to the type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


def reference(table, positions, x, backward):
    """(turned, bound) in binary64, from the table's fractions of a turn by whole-number arithmetic."""
    rot = table.rot_dim
    frac = torch.tensor([[((int(p) * f) % (1 << 64)) / 2.0 ** 64 for f in table.fractions] for p in positions], dtype=torch.float64).reshape(-1, rot // 2)
    cos, sin = (f(2 * math.pi * frac).unsqueeze(1) * table.magnitude for f in (torch.cos, torch.sin))
    if backward:
        sin = -sin
    x = x.double()
    y, bound = x.clone(), torch.zeros_like(x)
    index = torch.arange(rot)
    first, second = (index[0::2], index[1::2]) if table.interleaved else (index[:rot // 2], index[rot // 2:])
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    both = (a.abs() + b.abs()) * table.magnitude * (2.0 ** -21 + 2.0 ** -23)
    bound[..., first] = bound[..., second] = both
    return y, bound


def check(got, table, positions, x, before, backward=False):
    live = [i for i, p in enumerate(positions.tolist()) if p >= 0]
    pad = [i for i, p in enumerate(positions.tolist()) if p < 0]
    got, x, before = got.cpu(), x.cpu(), before.cpu()
    assert torch.equal(got[pad], before[pad])
    y, bound = reference(table, positions[live].tolist(), x[live], backward)
    step = torch.finfo(got.dtype).eps / 2
    tol = bound * (1 + step) + step * y.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    tol[..., table.rot_dim:] = 0
    assert not bool(((got[live].double() - y).abs() > tol).any())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,kv_heads,dim,rot", [
    (1, 1, 1, 64, 64), (3, 4, 2, 128, 128), (65, 32, 8, 128, 128), (17, 5, 5, 80, 64), (9, 3, 1, 256, 256), (40, 8, 2, 96, 48), (7, 2, 1, 33, 2), (5, 2, 2, 100, 50),
    (33, 7, 1, 72, 36), (21, 40, 8, 128, 16), (300, 6, 2, 64, 8), (2, 64, 0, 128, 128), (700, 32, 8, 128, 128)])
def test_turns_match_the_definition(B, dtype, interleaved, n, heads, kv_heads, dim, rot):
    g = torch.Generator().manual_seed(n + dim)
    table = B.RotaryTable(rot, interleaved=interleaved)
    positions = torch.randint(0, 1 << 17, (n,), generator=g)
    if n > 2:
        positions[n // 2] = -1
        positions[0] = 0
    both = (torch.randn(n, heads + 2 * kv_heads, dim, generator=g) * 3).to(TD[dtype]).cuda()
    q, k = both[:, :heads], both[:, heads:heads + kv_heads] if kv_heads else None
    backward = n % 2 == 1
    outs = [torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") if t is not None else None for t in (q, k)]
    untouched = both.clone()
    B.rotary_launch(table, positions.cuda(), q, k, *outs, backward=backward)
    assert torch.equal(both, untouched)
    for x, out in zip((q, k), outs):
        if x is not None:
            check(out, table, positions, x, torch.full_like(x, 7.0), backward)
    # in place, inside the fused tensor: nothing else of it moves
    B.rotary_launch(table, positions.cuda(), q, k, backward=backward)
    for at, out in ((slice(0, heads), outs[0]), (slice(heads, heads + kv_heads), outs[1])):
        if out is not None:
            want = out.clone()
            want[positions < 0] = untouched[:, at][positions < 0]
            assert torch.equal(both[:, at], want)
    assert torch.equal(both[:, heads + kv_heads:], untouched[:, heads + kv_heads:])


@pytest.mark.parametrize("scaling,kw", [("linear", {}), ("ntk", {}), ("bands", dict(original_len=8192, low_turns=1.0, high_turns=4.0)),
                                        ("yarn", dict(original_len=4096, fast_turns=32.0, slow_turns=1.0)), ("yarn", dict(original_len=4096, magnitude=1.25))])
@pytest.mark.parametrize("far", [1 << 10, 1 << 20, 1 << 44])
def test_scaled_frequencies_and_far_positions(B, scaling, kw, far):
    g = torch.Generator().manual_seed(3)
    table = B.RotaryTable(128, base=500000.0, scaling=scaling, factor=8.0, **kw)
    positions = torch.randint(0, far, (50,), generator=g)
    positions[0] = far - 1
    q = torch.randn(50, 4, 128, generator=g).cuda()
    out = torch.empty_like(q)
    B.rotary_launch(table, positions.cuda(), q, q_out=out)
    check(out, table, positions, q, q)


@pytest.mark.parametrize("offset", [1, 2, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_slices_off_the_vector_alignment(B, offset, dtype):
    table = B.RotaryTable(64)
    base = torch.randn(30, 6, 64 + 24, device="cuda").to(TD[dtype])
    out = torch.zeros(30, 6, 64 + 24, device="cuda", dtype=TD[dtype])
    positions = torch.arange(30)
    q = base[..., offset:offset + 64]
    B.rotary_launch(table, positions.cuda(), q, q_out=out[..., 24 - offset:88 - offset])
    check(out[..., 24 - offset:88 - offset], table, positions, q, q)
    out[..., 24 - offset:88 - offset] = 0
    assert not bool(out.any())


def test_head_major_tensors(B):
    table = B.RotaryTable(128, interleaved=True)
    base = torch.randn(8, 50, 128, device="cuda", dtype=torch.bfloat16)
    q = base.permute(1, 0, 2)  # [tokens, heads, dim], the heads outermost
    positions, before = torch.arange(50), q.clone()
    B.rotary_launch(table, positions.cuda(), q)
    check(q, table, positions, before, before)


def test_the_gradient_is_that_of_the_turn(B):
    """<g, R x> = <R' g, x> for the backward form R', in binary32: the sums differ by their roundings alone."""
    for interleaved in (False, True):
        table = B.RotaryTable(96, scaling="yarn", factor=4.0, original_len=2048, interleaved=interleaved)
        positions = torch.randint(0, 100000, (64,)).cuda()
        x, g = torch.randn(2, 64, 3, 128, device="cuda").unbind(0)
        y, gx = torch.empty_like(x), torch.empty_like(x)
        B.rotary_launch(table, positions, x.contiguous(), q_out=y)
        B.rotary_launch(table, positions, g.contiguous(), q_out=gx, backward=True)
        left, right = (g.double() * y.double()).sum(-1), (gx.double() * x.double()).sum(-1)
        bound = 2.0 ** -20 * 2 * (x.double().norm(dim=-1) * g.double().norm(dim=-1)) * table.magnitude
        assert not bool(((left - right).abs() > bound).any())
        # and against differences along a random direction: the turn is linear, so a difference of any length is its gradient
        h = torch.randn_like(x)
        y2 = torch.empty_like(x)
        B.rotary_launch(table, positions, (x + h).contiguous(), q_out=y2)
        along, want = ((y2 - y).double() * g.double()).sum(-1), (gx.double() * h.double()).sum(-1)
        size = (x.double().norm(dim=-1) + 2 * h.double().norm(dim=-1)) * g.double().norm(dim=-1) * table.magnitude
        assert not bool(((along - want).abs() > 2.0 ** -19 * size).any())


def test_infinities_stay_in_their_pairs(B):
    table = B.RotaryTable(64)
    q = torch.randn(4, 2, 64, device="cuda")
    q[1, 0, 3] = math.inf
    q[2, 1, 40] = math.nan
    out = torch.empty_like(q)
    B.rotary_launch(table, torch.arange(1, 5, device="cuda"), q, q_out=out)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1, 0, 3] = want[1, 0, 35] = want[2, 1, 8] = want[2, 1, 40] = True
    assert torch.equal(bad, want)


def test_streams_graphs_and_no_tokens(B):
    table = B.RotaryTable(128)
    q = torch.randn(64, 8, 128, device="cuda", dtype=torch.bfloat16)
    positions = torch.arange(64, device="cuda")
    want = torch.empty_like(q)
    B.rotary_launch(table, positions, q, q_out=want)
    side = torch.cuda.Stream()
    got = torch.zeros_like(q)
    side.wait_stream(torch.cuda.current_stream())
    B.rotary_launch(table, positions, q, q_out=got, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    got.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rotary_launch(table, positions, q, q_out=got)
    for step in range(3):
        positions += 5
        graph.replay()
        B.rotary_launch(table, positions, q, q_out=want)
        assert torch.equal(got, want)
    B.rotary_launch(table, positions[:0], q[:0])
    B.rotary_launch(table, positions, q[:, :0])


def test_refusals(B):
    table = B.RotaryTable(128)
    q, positions = torch.randn(4, 2, 128, device="cuda"), torch.arange(4, device="cuda")
    for bad in (dict(positions=positions.int()), dict(positions=positions[:3]), dict(q=q[0]), dict(q=q.cpu()), dict(q=q.double()), dict(q=q.transpose(1, 2)),
                dict(q_out=q.bfloat16()), dict(q_out=q[:3]), dict(k=q[:, :, :64]), dict(k=q.half()), dict(k_out=q), dict(q_out=q[:, :1].expand(4, 2, 128))):
        args = dict(positions=positions, q=q)
        args.update(bad)
        with pytest.raises((ValueError, B.TunerError)):
            B.rotary_launch(table, **args)
    with pytest.raises(B.TunerError):
        B.rotary_launch(table, positions, q[..., :64])  # heads smaller than what is turned
