"""Frequencies of rotary positions and the refusals of their entry points, without a GPU (pointers are numbers that nothing follows)."""
import ctypes
import math

import pytest

from paper_2601_12698_b200 import binding as B

P = 1 << 20


def _spec(**kw):
    d = dict(base=10000.0, factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=4.0, fast_turns=32.0, slow_turns=1.0, rot_dim=128, scaling=B.RT_ROTARY_NONE)
    d.update(kw)
    return B.rt_rotary_spec(**d)


def _frequencies(spec):
    out, m = (ctypes.c_uint64 * 128)(), ctypes.c_float()
    assert B.lib.rotary_frequencies(ctypes.byref(spec), out, ctypes.byref(m)) == B.RT_OK
    return list(out)[:spec.rot_dim // 2], m.value


def _theta(j, rot, kind, p):
    """The definition, a pair at a time."""
    base = p["base"] * p["factor"] ** (rot / (rot - 2)) if kind == B.RT_ROTARY_NTK else p["base"]
    theta = base ** (-2 * j / rot)
    if kind == B.RT_ROTARY_LINEAR:
        return theta / p["factor"]
    if kind == B.RT_ROTARY_BANDS:
        turns = p["original_len"] * theta / (2 * math.pi)
        if turns <= p["low_turns"]:
            return theta / p["factor"]
        if turns >= p["high_turns"]:
            return theta
        w = (turns - p["low_turns"]) / (p["high_turns"] - p["low_turns"])
        return w * theta + (1 - w) * theta / p["factor"]
    if kind == B.RT_ROTARY_YARN:
        pair = lambda n: rot * math.log(p["original_len"] / (2 * math.pi * n)) / (2 * math.log(base))
        first, last = max(0, math.floor(pair(p["fast_turns"]))), min(rot - 1, math.ceil(pair(p["slow_turns"])))
        if j <= first:
            return theta
        if j >= last:
            return theta / p["factor"]
        w = (j - first) / (last - first)
        return theta * (1 - w) + theta / p["factor"] * w
    return theta


@pytest.mark.parametrize("kind", range(5))
@pytest.mark.parametrize("rot,base,factor", [(128, 10000.0, 8.0), (64, 500000.0, 4.0), (96, 1e6, 32.0), (4, 10000.0, 2.0), (256, 10000.0, 0.5), (2, 100.0, 3.0)])
def test_frequencies_follow_the_definition(kind, rot, base, factor):
    if kind == B.RT_ROTARY_NTK and rot == 2:
        return
    p = dict(base=base, factor=factor, original_len=8192.0, low_turns=1.0, high_turns=4.0, fast_turns=32.0, slow_turns=1.0)
    got, magnitude = _frequencies(_spec(rot_dim=rot, scaling=kind, **p))
    for j, turns in enumerate(got):
        want = _theta(j, rot, kind, p) / (2 * math.pi)
        # a few roundings of 2^-53 each in powers and logarithms, times exponents of at most ln(base') of magnitude 20
        assert abs(turns * 2.0 ** -64 - (want - math.floor(want))) <= 64 * 2.0 ** -53 * want + 2.0 ** -63
    assert magnitude == pytest.approx(0.1 * math.log(factor) + 1 if kind == B.RT_ROTARY_YARN else 1.0, rel=2.0 ** -23)


@pytest.mark.parametrize("change", [
    {"rot_dim": 0}, {"rot_dim": 3}, {"rot_dim": 258}, {"scaling": -1}, {"scaling": 5}, {"base": 1.0}, {"base": math.nan}, {"base": math.inf},
    {"scaling": 1, "factor": 0.0}, {"scaling": 1, "factor": math.inf}, {"scaling": 2, "rot_dim": 2}, {"scaling": 3, "original_len": 0.0},
    {"scaling": 3, "low_turns": 4.0}, {"scaling": 3, "low_turns": 0.0}, {"scaling": 4, "fast_turns": 1.0}, {"scaling": 4, "slow_turns": -1.0},
    {"scaling": 4, "original_len": math.nan}])
def test_frequency_refusals(change):
    out, m = (ctypes.c_uint64 * 128)(), ctypes.c_float()
    assert B.lib.rotary_frequencies(ctypes.byref(_spec(**change)), out, ctypes.byref(m)) == B.RT_ERR_SHAPE
    assert B.lib.rt_last_error()
    assert B.lib.rotary_frequencies(None, out, ctypes.byref(m)) == B.RT_ERR_NULL


def _call(rotary=None, tokens=5, dim=128, q=(P, 512, 128, P, 512, 128, 4), k=(P, 256, 128, P, 256, 128, 2), dtype=0, positions=P):
    r = B.rt_rotary(P, 128, 0, 0, 1.0) if rotary is None else rotary
    sides = (B.rt_rotary_side * 2)(*[B.rt_rotary_side(s[0], s[3], s[1], s[2], *s[4:]) for s in (q, k)])
    return B.lib.rotary_launch(ctypes.byref(r), positions, tokens, dim, ctypes.cast(sides, ctypes.c_void_p), dtype, None)


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), "RT_ERR_SHAPE"), (dict(dim=0), "RT_ERR_SHAPE"), (dict(dim=257), "RT_ERR_SHAPE"), (dict(dim=64), "RT_ERR_SHAPE"), (dict(dtype=3), "RT_ERR_DTYPE"),
    (dict(rotary=B.rt_rotary(P, 0, 0, 0, 1.0)), "RT_ERR_SHAPE"), (dict(rotary=B.rt_rotary(P, 7, 0, 0, 1.0)), "RT_ERR_SHAPE"),
    (dict(rotary=B.rt_rotary(None, 64, 0, 0, 1.0)), "RT_ERR_NULL"), (dict(positions=None), "RT_ERR_NULL"), (dict(positions=P + 4), "RT_ERR_ALIGN"),
    (dict(q=(None, 512, 128, P, 512, 128, 4)), "RT_ERR_NULL"), (dict(k=(P, 256, 128, None, 256, 128, 2)), "RT_ERR_NULL"),
    (dict(q=(P + 1, 512, 128, P, 512, 128, 4)), "RT_ERR_ALIGN"), (dict(q=(P, -512, 128, P, 512, 128, 4)), "RT_ERR_SHAPE"),
    (dict(q=(P, 512, 128, P, 0, 128, 4)), "RT_ERR_SHAPE"), (dict(q=(P, 512, 128, P, 512, 0, 4)), "RT_ERR_SHAPE"), (dict(q=(P, 512, 128, P, 512, 128, -4)), "RT_ERR_SHAPE"),
    (dict(k=(P, 256, 128, P, 512, 128, 2)), "RT_ERR_SHAPE")])  # the last: in place with two strides
def test_launch_refusals(kw, status):
    assert _call(**kw) == getattr(B, status)
    assert B.lib.rt_last_error()


def test_nothing_to_do_is_no_error():
    none = (None, 0, 0, None, 0, 0, 0)
    assert _call(q=none, k=none) == B.RT_OK
    assert _call(tokens=0, positions=None) == B.RT_OK
    assert B.lib.rotary_launch(None, P, 5, 128, P, 0, None) == B.RT_ERR_NULL
    assert B.lib.rotary_launch(ctypes.byref(B.rt_rotary(P, 128, 0, 0, 1.0)), P, 5, 128, None, 0, None) == B.RT_ERR_NULL
    with pytest.raises(ValueError):
        B.RotaryTable(64, scaling="other", device="cpu")
    with pytest.raises(B.TunerError):
        B.RotaryTable(63, device="cpu")


@pytest.mark.parametrize("q,k", [((P, 512, 128, P, 512, 128, 4), (P, 256, 128, P, 256, 128, 2)), ((P, 512, 128, P + 4096, 512, 128, 4), (P + 4096, 256, 128, P + 4096, 256, 128, 2)),
                                 ((P, 512, 128, P, 512, 128, 4), (P + 4096, 256, 128, P, 256, 128, 2))])
def test_sides_that_are_one_another_are_refused(q, k):
    assert _call(q=q, k=k) == B.RT_ERR_SHAPE and "overlap" in B.lib.rt_last_error().decode()
