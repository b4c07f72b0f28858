"""Far positions against angles from the definition in 60 digits, not from the library's own fractions.

Tolerance: that of test_gpu_rotary.py for the cosines, sines, products and the rounding, and an angle that is off by position * 2^-63 turns."""
import math
from decimal import localcontext

import pytest
import torch

import rotary_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


@pytest.mark.parametrize("kw", [dict(), dict(scaling="ntk", factor=8.0), dict(scaling="bands", factor=8.0, original_len=8192.0), dict(scaling="yarn", factor=8.0, original_len=4096.0)])
@pytest.mark.parametrize("far", [1 << 17, 1 << 30, 1 << 37, 1 << 44])
def test_far_positions_follow_the_definition(B, kw, far):
    rot, base = 128, 500000.0
    g = torch.Generator().manual_seed(far % 1000)
    positions = torch.randint(far // 2, far, (40,), generator=g)
    positions[0] = far - 1
    x = torch.randn(40, 3, rot, generator=g)
    table = B.RotaryTable(rot, base=base, **kw)
    out = torch.empty_like(x.cuda())
    B.rotary_launch(table, positions.cuda(), x.cuda(), q_out=out)
    with localcontext() as c:
        c.prec = 60
        angle = [[2 * math.pi * float(int(p) * t % 1) for t in R.turns(rot, base, **kw)] for p in positions]
    angle = torch.tensor(angle, dtype=torch.float64)[:, None]
    cos, sin = angle.cos() * table.magnitude, angle.sin() * table.magnitude
    a, b = x.double().chunk(2, -1)
    want = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    size = ((a.abs() + b.abs()) * table.magnitude).repeat(1, 1, 2)
    tol = size * (2.0 ** -21 + 2.0 ** -23 + 2 * math.pi * positions.double()[:, None, None] * 2.0 ** -63) + 2.0 ** -24 * want.abs()
    assert not bool(((out.cpu().double() - want).abs() > tol).any())
