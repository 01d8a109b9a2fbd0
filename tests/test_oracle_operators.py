"""CPU tests of the sampling reference's masses: the definition of fgd.h, step
by step in whole numbers."""

from fractions import Fraction

import numpy as np

from oracle import operators as ref


def _round_f32(x):
    """The float32 nearest to a positive Fraction, ties to even."""
    e = 0
    while x >= 2:
        x, e = x / 2, e + 1
    while x < 1:
        x, e = x * 2, e - 1
    n = x * 2 ** 23
    whole = n.numerator // n.denominator
    rest = n - whole
    if rest > Fraction(1, 2) or (rest == Fraction(1, 2) and whole % 2):
        whole += 1
    return Fraction(whole) * Fraction(2) ** (e - 23)


def test_masses_by_their_definition():
    rng = np.random.default_rng(1)
    w = np.exp2(-34 * rng.random(4000)).astype(np.float32)
    half = np.float32(2.0 ** -32)  # a mass of one half
    w = np.concatenate([w, [1, 0.5, half, np.nextafter(half, np.float32(0)), np.nextafter(half, np.float32(1)), 0]])
    got = ref.mass_of(w)
    for x, m in zip(w, got):
        want = _round_f32(Fraction(float(x)) * 2 ** 31 + Fraction(1, 2))
        assert m == want.numerator // want.denominator


def test_ties_go_to_the_even_mass():
    n = np.arange(2 ** 23, 2 ** 23 + 1001)
    assert np.array_equal(ref.mass_of(n * 2.0 ** -31), n + n % 2)
    n = np.arange(2 ** 24 - 1000, 2 ** 24 + 1)
    assert np.array_equal(ref.mass_of(n * 2.0 ** -31), n + n % 2)
    n = np.arange(2 ** 22, 2 ** 22 + 1000)  # below, every sum is exact
    assert np.array_equal(ref.mass_of(n * 2.0 ** -31), n)
    assert np.array_equal(ref.mass_of((n + 0.5) * 2.0 ** -31), n + 1)
