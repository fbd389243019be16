"""The frequencies of the rotation against the definitions in 60 digits, and the angle that a position makes of them (no GPU needed)."""
import math
from decimal import Decimal as D
from decimal import getcontext

import numpy as np
import pytest

getcontext().prec = 60


def _pi():
    """By Machin's formula."""
    def arctan_of_1_over(n):
        total, power, k = D(0), D(1) / n, 0
        while abs(power) > D(10) ** -58:
            total += power / (2 * k + 1) * (-1) ** k
            power /= n * n
            k += 1
        return total
    return 4 * (4 * arctan_of_1_over(5) - arctan_of_1_over(239))


def exact_turns(rot, base, scaling="none", factor=1.0, low=1.0, high=32.0, original=8192.0):
    """Turns a position of every pair."""
    base, factor, low, high, original, two_pi, out = D(base), D(factor), D(low), D(high), D(original), 2 * _pi(), []
    for i in range(rot // 2):
        w = (base.ln() * -2 * i / rot).exp()
        if scaling == "linear":
            w /= factor
        elif scaling == "bands":
            keep = min(max((original * w / two_pi - low) / (high - low), D(0)), D(1))
            w *= keep + (1 - keep) / factor
        elif scaling == "yarn":
            pair = lambda turns: rot * (original / (two_pi * turns)).ln() / (2 * base.ln())  # noqa: E731
            first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
            ramp = min(max(D(i - first) / max(D(last - first), D("0.001")), D(0)), D(1))
            w *= 1 - ramp + ramp / factor
        out.append(w / two_pi)
    return out


CASES = [("none", 10000.0, {}), ("none", 500000.0, {}), ("none", 1.5, {}), ("linear", 10000.0, {"factor": 4.0}), ("linear", 10000.0, {"factor": 3.0}),
         ("bands", 500000.0, {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192}), ("yarn", 10000.0, {"factor": 32.0, "low": 1.0, "high": 32.0, "original": 4096}),
         ("yarn", 1000000.0, {"factor": 5.0, "low": 1.0, "high": 32.0, "original": 32768})]


def test_pi():
    assert abs(float(_pi()) - math.pi) < 1e-15 and str(_pi())[:22] == "3.14159265358979323846"


@pytest.mark.parametrize("rot", [2, 24, 64, 128, 256])
@pytest.mark.parametrize("scaling,base,kw", CASES)
def test_frequencies_are_off_by_two_steps_at_most(lib, rot, scaling, base, kw):
    """A step is 2^-64 of a turn.  Half of one is the last rounding; before it a frequency, at most 1 / (2 pi) of a turn, passes through
    fewer than ten operations of 64 bits, each off by 2^-64 of its value or, the power, by 2^-63: 1.8 steps.  An angle is then off
    by 2^-31 turns at the farthest position."""
    got = lib.new_rotary_table(rot, base, scaling, **kw, device="cpu").freq.numpy().view(np.uint64)
    for i, (g, want) in enumerate(zip(got.tolist(), exact_turns(rot, base, scaling, **kw))):
        assert abs(g - want * 2 ** 64) <= D("2.3"), (i, g - want * 2 ** 64)
        for pos in (2 ** 24, 2 ** 31 - 1):
            turn = (g * pos) % 2 ** 64
            off = (D(turn) / 2 ** 64 - want * pos + D("0.5")) % 1 - D("0.5")
            off = off + 1 if off < D("-0.5") else off
            assert abs(off) <= D(pos) * D("2.3") / 2 ** 64
