"""The fractions of a turn against their definition in 60 digits: to the last of their 64 bits, since every position multiplies their error."""
from decimal import Decimal, localcontext

import pytest

import rotary_reference as R
from paper_2601_12698_b200 import binding as B

SPECS = [dict(), dict(scaling="linear", factor=3.0), dict(scaling="ntk", factor=8.0), dict(scaling="bands", factor=8.0, original_len=8192.0),
         dict(scaling="yarn", factor=8.0, original_len=4096.0), dict(scaling="yarn", factor=40.0, original_len=4096.0, fast_turns=30.0), dict(scaling="linear", factor=0.1)]


@pytest.mark.parametrize("kw", SPECS)
@pytest.mark.parametrize("rot,base", [(128, 10000.0), (128, 500000.0), (64, 1e6), (256, 10000.0), (48, 1234.5), (4, 7.0)])
def test_fractions_are_right_to_their_last_bit(kw, rot, base):
    """One unit: half of it is the rounding to 64 bits.  The rest is 1 / 2 pi = 0.16 times theta times what powers and the ramp lose in 64 bits
    of mantissa: 2^-64 each for the power, the division by 2 pi and up to six operations of the ramp, and 2^-64 y e^-y <= 0.37 * 2^-64 for the
    exponent, y = 2 j ln(base) / rot: less than 0.16 * (8 + 0.37) / 2 more where theta <= 1."""
    got = B.RotaryTable(rot, base=base, device="cpu", **kw).fractions
    with localcontext() as c:
        c.prec = 60
        for j, (f, want) in enumerate(zip(got, R.turns(rot, base, **kw))):
            off = (Decimal(f) / 2 ** 64 - want) % 1
            off = min(abs(off), abs(1 - abs(off)))
            theta = max(1, want * R.TWO_PI)
            assert off * 2 ** 64 <= Decimal("1.2") * theta, (j, float(off * 2 ** 64))
