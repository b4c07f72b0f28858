"""Frequencies of rotary positions from their definition in 60 decimal digits.  Nothing here comes from the library."""
from __future__ import annotations

from decimal import ROUND_CEILING, ROUND_FLOOR, Decimal, localcontext

TWO_PI = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640629")


def turns(rot, base, scaling="none", factor=1.0, original_len=0.0, low_turns=1.0, high_turns=4.0, fast_turns=32.0, slow_turns=1.0):
    """What every pair makes of a full turn per position, as Decimals that need not be below one."""
    with localcontext() as c:
        c.prec = 60
        base, factor, original, low, high, fast, slow = (Decimal(x) for x in (base, factor, original_len, low_turns, high_turns, fast_turns, slow_turns))
        if scaling == "ntk":
            base *= (factor.ln() * rot / (rot - 2)).exp()
        out = []
        for j in range(rot // 2):
            theta = (base.ln() * -2 * j / rot).exp()
            if scaling == "linear":
                theta /= factor
            if scaling == "bands":
                keep = min(max((original * theta / TWO_PI - low) / (high - low), Decimal(0)), Decimal(1))
                theta = theta * keep + theta / factor * (1 - keep)
            if scaling == "yarn":
                pair = lambda n: rot * (original / (TWO_PI * n)).ln() / (2 * base.ln())
                first = max(Decimal(0), pair(fast).to_integral_value(ROUND_FLOOR))
                last = min(Decimal(rot - 1), pair(slow).to_integral_value(ROUND_CEILING))
                divided = min(max((j - first) / max(last - first, Decimal("0.001")), Decimal(0)), Decimal(1))
                theta = theta / factor * divided + theta * (1 - divided)
            out.append(theta / TWO_PI)
        return out
