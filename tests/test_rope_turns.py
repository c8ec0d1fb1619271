"""The pairs' frequencies against their formulas in 80 decimal digits: each is f_i / 2 pi as a 64-bit fraction of a turn, within
one unit of the exact one for frequencies of up to 2^30 turns a token (half a unit is the rounding, 2^-95 of the frequency
what it is formed with)."""
from decimal import ROUND_CEILING, ROUND_FLOOR, Decimal, getcontext

import numpy as np
import pytest

from paper_2607_02963_gb300 import binding as B

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def exact_turns(rotary, theta, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=4.0):
    """f_i / 2 pi, as Decimals."""
    getcontext().prec = 80
    t, s, length, lo, hi = (Decimal(x) for x in (theta, factor, original_len, low, high))
    if scaling == "base":
        t = t * (s.ln() * rotary / (rotary - 2)).exp()
    out = []
    if scaling == "index":
        def index(n, way):
            x = rotary * (length / (2 * PI * n)).ln() / (2 * t.ln())
            return min(max(x.to_integral_value(way), Decimal(0)), Decimal(rotary - 1))
        a, b = index(hi, ROUND_FLOOR), index(lo, ROUND_CEILING)
    log = t.ln()
    for i in range(rotary // 2):
        f = (log * -2 * i / rotary).exp()
        g = Decimal(1)
        if scaling == "linear":
            g = Decimal(0)
        if scaling == "turns":
            g = (length * f / (2 * PI) - lo) / (hi - lo)
        if scaling == "index":
            g = 1 - (i - a) / max(b - a, Decimal("0.001"))
        g = min(max(g, Decimal(0)), Decimal(1))
        out.append(f * (g + (1 - g) / s) / (2 * PI))
    return out


SPECS = [dict(theta=1e6), dict(theta=1e4), dict(theta=500.0), dict(theta=1.0), dict(theta=0.001), dict(theta=1e300),
         dict(theta=1e6, scaling="linear", factor=4.0), dict(theta=1e4, scaling="linear", factor=0.01),
         dict(theta=1e4, scaling="linear", factor=3e-9), dict(theta=1e6, scaling="base", factor=8.0),
         dict(theta=1e4, scaling="base", factor=0.1), dict(theta=1e4, scaling="base", factor=1e300),
         dict(theta=5e5, scaling="turns", factor=8.0, original_len=8192.0, low=1.0, high=4.0),
         dict(theta=1e6, scaling="turns", factor=0.3, original_len=32768.0, low=-1.0, high=1000.5),
         dict(theta=1e4, scaling="index", factor=4.0, original_len=4096.0, low=1.0, high=32.0),
         dict(theta=1e6, scaling="index", factor=40.0, original_len=131072.0, low=0.5, high=0.6)]


@pytest.mark.parametrize("rotary", [4, 54, 64, 128])
@pytest.mark.parametrize("spec", SPECS, ids=lambda s: "-".join(f"{v:g}" if isinstance(v, float) else v for v in s.values()))
def test_each_turn_is_within_a_unit(padlib, spec, rotary):
    got = B.Rope(128, rotary, **spec).turns.turn[:rotary // 2]
    for i, (g, want) in enumerate(zip(got, exact_turns(rotary, **spec))):
        off = abs(Decimal(g) - want % 1 * 2 ** 64)
        assert min(off, 2 ** 64 - off) <= 1, f"pair {i}: {float(off)} units"


def test_a_magnitude_beyond_32_bits_is_refused(padlib):
    B.Rope(128, magnitude=float(np.finfo(np.float32).max))
    for bad in (3.5e38, -1e300):
        with pytest.raises(B.PadError, match="magnitude"):
            B.Rope(128, magnitude=bad)
