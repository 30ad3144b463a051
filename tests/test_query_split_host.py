"""What is left of a query that attention over the cache in 4 bits takes as three numbers of 6 bits, by enumeration.

32 channels share 2^e, the least with max |q| <= 7.5 * 2^e and e >= -118; the terms are the nearest numbers of e2m3 (steps of
1/8 to 2, of 1/4 to 4, of 1/2 to 7.5; ties to even) at 2^e, 2^(e-4) and 2^(e-9), each of what those before it left.  A bf16
number leaves no more than 2^-8 of 2^e to the third, whose step there is 2^-12: 2^-13 of 2^e is what can be lost, and the
largest of the 32 is above 3.75 * 2^e (where e is not held at -118): 2^-14.9 of it.  Numbers of 2^-5 of 2^e or more have no bit
below 2^-12 of it and lose nothing: those are all that are no smaller than 1/64 of the largest."""
import numpy as np
import pytest

LOST = 2.0 ** -14.9        # of the largest of 32 channels
EXACT = 1 / 64             # of it, and above: nothing is lost
SMALL = 2.0 ** -131        # and what small groups lose


def six(x):
    """float64, |x| <= 7.5 -> the nearest number of e2m3."""
    a = np.abs(x)
    step = np.where(a < 2, 0.125, np.where(a < 4, 0.25, 0.5))
    return np.copysign(np.minimum(np.round(a / step) * step, 7.5), x)


def exponent(largest):
    """e of groups whose largest magnitude is given (bf16, not 0)."""
    m, e = np.frexp(largest)                                  # m in [1/2, 1)
    return np.maximum(np.where(m <= 0.9375, e - 3, e - 2), -118)


def split(q):
    """float64 [..., 32] of bf16 numbers -> the sums of their three terms."""
    largest = np.max(np.abs(q), axis=-1, keepdims=True)
    unit = np.exp2(exponent(np.where(largest > 0, largest, 1.0)).astype(np.float64))
    left, total = q / unit, np.zeros(q.shape)
    for s in (1.0, 2.0 ** -4, 2.0 ** -9):
        assert np.all(np.abs(left) <= 7.5 * s)
        term = six(left / s) * s
        left, total = left - term, total + term
    return total * unit


def bf16(lo, hi):
    """All positive bf16 numbers of the exponents lo .. hi - 1 (below -126: those of -126 that have none of their own)."""
    m = 1 + np.arange(128) / 128.0
    x = np.concatenate([m * 2.0 ** e for e in range(max(lo, -126), hi)])
    return np.concatenate([np.arange(1, 128) * 2.0 ** -133, x]) if lo < -126 else x


@pytest.mark.parametrize("e", [0, 1, 126, 127, -100, -115, -116, -117, -118, -119, -125, -126])
def test_bound(e):
    """Every largest number of an exponent beside every number that is not above it."""
    worst = 0.0
    below = bf16(max(e - 40, -127), e + 1)
    for top in bf16(e, e + 1):
        v = below[below <= top]
        q = np.concatenate([v, [0.0] * (-len(v) % 31)]).reshape(-1, 31)
        q = np.concatenate([q, np.full((len(q), 1), top)], -1)
        lost = np.abs(split(q) - q)
        held = exponent(top) == -118
        assert np.all(lost <= max(LOST * top, SMALL if held else 0.0))
        if not held:
            assert not lost[q >= EXACT * top].any()
            worst = max(worst, float(lost.max() / top))
    # and it is no larger than it has to be
    assert worst == 0.0 if e <= -117 else worst > 0.99 * 2.0 ** -13 / 3.765625


def test_a_number_of_the_bound():
    """3.765625 and the 128th part of it, which is off by more than 2^-15 of the largest."""
    q = np.zeros((1, 32))
    q[0, :2] = 3.765625, 3.765625 / 128
    lost = np.abs(split(q) - q)[0]
    assert lost[0] == 0.0 and lost[1] == 2.0 ** -13 > 2.0 ** -15 * 3.765625


def test_signs_and_zeros():
    rng = np.random.default_rng(1)
    x = bf16(-12, 2)
    q = rng.choice(x, (500, 32)) * rng.choice([-1, 1], (500, 32))
    assert np.array_equal(split(-q), -split(q))
    assert not split(np.zeros((2, 32))).any()
