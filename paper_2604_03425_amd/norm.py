"""The integers of ckks_rmsnorm for a range of the mean square: where Newton's steps for 1 / sqrt(m) start and how their scales follow
from the primes that are divided away. Host arithmetic, in double precision."""
import math


def _step(w):
    """What a step makes of y sqrt(m)."""
    return w * (3.0 - w * w) / 2.0


def _start(rho, iterations):
    """(alpha, beta) of the start y = alpha - beta m on [rho, 1], and the lowest y sqrt(m) after the steps. y sqrt(m) is the same at both
    ends and highest between them; a step maps [0, 1] upwards and what is above 1 below it, so that the best line is the one whose two
    extremes a step makes equal."""
    r = math.sqrt(rho)
    low, high = r + rho, 2.0 / 3.0 * (1.0 + r + rho) * math.sqrt((1.0 + r + rho) / 3.0)   # extremes for beta = 1
    if iterations == 0:
        beta = 2.0 / (low + high)
        return beta * (1.0 + r + rho), beta, low * beta
    a, b = 1.0 / high, math.sqrt(3.0) / high
    for _ in range(200):
        beta = 0.5 * (a + b)
        if _step(low * beta) < _step(high * beta):
            a = beta
        else:
            b = beta
    w = low * beta
    for _ in range(iterations):
        w = _step(w)
    return beta * (1.0 + r + rho), beta, w


def rmsnorm_plan(q, nlimbs, scale, components, lo, hi, iterations, eps=0.0):
    """Arguments of ckks_rmsnorm for inputs of nlimbs limbs at `scale` (after the residual's addition) with `components` components a
    lane, where the mean square (eps included) lies in [lo, hi]. q: the context's main primes. Returns a dict:
        square, eps, start, factors   the call's integers
        scale      of the factor 1 / sqrt(mean square + eps): the output's scale is this times the input's (times gain's scale over
                   q[nlimbs - 1 - 2 iterations], the prime that its product with the input is rescaled by)
        error      the largest relative error of that factor on the range, without noise
    The scale of the mean square, components scale^2 / q[nlimbs - 1], may be up to about half of the primes' cube root of product: a larger
    one is refused, since a product can only raise it. The scales stay where they are while a step divides by primes of one size; a chain
    whose primes grow from step to step shrinks them, and one where an integer would be rounded by more than 2^-17 of itself is refused."""
    if not 0.0 < lo <= hi:
        raise ValueError("need 0 < lo <= hi")
    if iterations < 0 or nlimbs < 2 + 2 * iterations or nlimbs > len(q):
        raise ValueError("the norm takes 1 + 2 iterations limbs and leaves one or more")
    per_mean = components * float(scale) ** 2 / q[nlimbs - 1]       # scale of the mean square for square = 1
    if iterations:
        cube = float(q[nlimbs - 2]) ** 2 * q[nlimbs - 3]            # what the first step divides by
    else:
        cube = float(q[nlimbs - 2]) ** 3
    # The scale S of m = mean / unit and the start's S / beta stay what they are over the steps for 2 S^3 = beta^2 cube. `square` is an
    # integer, so the unit (hi or more) makes up for its rounding.
    def steady(unit):
        beta = _start(lo / unit, iterations)[1]
        return (cube * beta * beta / 2.0) ** (1.0 / 3.0)

    square = int(steady(hi) / (per_mean * hi))
    if square < 1:
        raise ValueError("the input's scale is too large for these primes")
    low, high = hi, 4.0 * hi
    for _ in range(100):                                            # steady(unit) / unit falls
        unit = 0.5 * (low + high)
        if steady(unit) > square * per_mean * unit:
            low = unit
        else:
            high = unit
    alpha, beta, least = _start(lo / unit, iterations)
    S = square * per_mean * unit
    y = S / beta
    numbers = dict(square=square, eps=round(S * eps / unit), start=round(alpha * y), factors=[])
    limbs = nlimbs - 1
    for _ in range(iterations):
        product = S * y ** 3 / float(q[limbs - 1]) ** 2             # scale of (m y) (y y)
        numbers["factors"].append(round(3.0 * product / y))
        y = 2.0 * product / q[limbs - 2]
        limbs -= 2
    # a factor off by e makes the step's result wrong by 3/2 e at most, which a further step squares
    if min([numbers["start"]] + numbers["factors"]) < 1 << 16:
        raise ValueError("the scales vanish over the steps: a step's primes are larger than those of the first one")
    if any(abs(v) >= 1 << 63 for v in [numbers["square"], numbers["eps"], numbers["start"]] + numbers["factors"]):
        raise ValueError("these scales take integers beyond 64 bits")
    return dict(numbers, scale=y * math.sqrt(unit), error=1.0 - least)
