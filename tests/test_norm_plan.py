"""The norm's integers on chains of primes of several sizes: what the call makes of them in exact arithmetic, against the stated error."""
import math
from fractions import Fraction

import pytest

from ckks_inputs import find_ntt_primes
from paper_2604_03425_amd.norm import rmsnorm_plan


def _chain(bits):
    q = []
    for b in bits:
        q += find_ntt_primes(b, 1, 13, exclude=set(q))
    return q


def _worst(q, plan, scale, components, lo, hi, points=33):
    """The largest relative error of the factor 1 / sqrt(mean square) over [lo, hi]."""
    worst, n = 0.0, len(q)
    for i in range(points):
        mean = lo * (hi / lo) ** (i / (points - 1))
        m = Fraction(plan["square"] * components) * Fraction(mean) * Fraction(scale) ** 2 / q[n - 1]
        y, limbs = plan["start"] - m, n - 1
        for f in plan["factors"]:
            u, w = m * y / q[limbs - 1], y * y / q[limbs - 1]
            y = (f * y - u * w) / q[limbs - 2]
            limbs -= 2
        worst = max(worst, abs(float(y) / plan["scale"] * math.sqrt(mean) - 1.0))
    return worst


CHAINS = [([50] * 8, 3), ([60] + [50] * 7, 3), ([36] * 8, 3), ([30] * 6, 2), ([45, 50] * 4, 3), ([60] * 3 + [50] * 5, 3), ([40, 50, 60, 60, 60], 1)]
SHRINKING = [([50] * 6 + [30, 50], 3), ([60] * 5 + [50] * 3, 3), ([60] * 4 + [45] * 4, 3), ([50] * 5 + [28] * 3, 3)]


@pytest.mark.parametrize("bits,steps", CHAINS)
@pytest.mark.parametrize("log_scale", [12, 18, 27])
def test_the_stated_error_holds(bits, steps, log_scale):
    """In double precision on the plan's side: 2^-40 of room for its own rounding, 3/2 2^-17 squared for the last but one factor's and
    3/2 e for the last one's, which is at most 2^-17 and 2^-30 here."""
    q, scale = _chain(bits), 2.0 ** log_scale
    try:
        plan = rmsnorm_plan(q, len(q), scale, 64, 1.0, 4.0, steps)
    except ValueError as e:
        # `square` is about the last prime times the cube root of what the first step divides by, over 64 scale^2: above 2^63 (50-bit primes
        # at 2^12, 60-bit ones at 2^18) or below 1 (30-bit ones at 2^27); and integers of a chain whose scales grow
        assert "beyond 64 bits" in str(e) or "too large" in str(e)
        return
    assert min(plan["factors"]) >= 1 << 16
    last = 0.75 / plan["factors"][-1]
    assert _worst(q, plan, scale, 64, 1.0, 4.0) <= plan["error"] + 2.0 ** -40 + (1.5 * 2.0 ** -17) ** 2 * 1.5 + last


@pytest.mark.parametrize("bits,steps", SHRINKING)
def test_chains_that_lose_their_scale_are_refused(bits, steps):
    """The first step divides by smaller primes than the later ones do: their factors would round to a few units or to nothing."""
    q = _chain(bits)
    with pytest.raises(ValueError, match="vanish"):
        rmsnorm_plan(q, len(q), 2.0 ** 12, 64, 1.0, 4.0, steps)
