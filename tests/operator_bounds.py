"""How far results of the dropout, norm and rotary operators may be from the float64 oracle, derived from their arithmetic.

A rounding to a type is off by at most half a step: U[dtype] of the value, or half of the smallest step where the value is
below the type's normal range.  float32 arithmetic adds U32 for every operation, of the terms that it works on."""
import numpy as np

from oracle import oracle as O

U32 = 2.0 ** -24
U = {"f32": U32, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
HALF_STEP_AT_ZERO = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}   # (float32: flushed subnormals are far below the terms' errors)
SMALLEST = 2.0 ** -126   # what float32 instructions may flush


def close(got, ref, dtype, error, what=""):
    """|got - ref| <= the rounding to `dtype` + `error` (float32 arithmetic, element by element)."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    error = np.broadcast_to(np.asarray(error, np.float64), ref.shape)
    bar = U[dtype] * (np.abs(ref) + error) + HALF_STEP_AT_ZERO[dtype] + error + SMALLEST
    off = np.abs(got - ref)
    assert got.shape == ref.shape, f"{what}: {got.shape} != {ref.shape}"
    assert np.isfinite(got).all(), f"{what}: non-finite"
    worst = int(np.argmax(off - bar))
    assert (off <= bar).all(), f"{what}: element {worst}: got {got.flat[worst]!r}, {ref.flat[worst]!r} expected, off by {off.flat[worst]:.3e} > {bar.flat[worst]:.3e}"


def activation_error(z, act):
    """Of act(z): its exponential and reciprocal are good to a few units in the last place, their argument to two roundings (|z| grows
    them: an argument's absolute error is a relative one of the exponential)."""
    return 0.0 if act == "none" else U32 * np.abs(z) * (12.0 + 4.0 * np.abs(z) * (1.0 + z * z))


def slope_error(z, act):
    """Of act'(z) = s + z s (1 - s) w with w = 1 or d(2u)/dz below 1.6 (1 + 0.14 z^2): each term's roundings and the argument's."""
    a = np.abs(z)
    return 0.0 if act == "none" else U32 * (12.0 + 8.0 * a * (1.0 + z * z)) * (1.0 + a)


def sum_error(terms_abs_sum, depth=64):
    """Of a float32 sum whose partial sums each round: `depth` roundings of the sum of magnitudes at most where a lane adds up to 64
    values and the rest goes pairwise."""
    return depth * U32 * terms_abs_sum


def eight_bit(q, s, n, n_error, what=""):
    """q (values) and its scale against the n that they stand for: q is the rounding of a quotient by that scale of a value within
    n_error of n, the quotient itself good to two units in the last place.  (Values of few bits often lie on a rounding border
    exactly, and the float32 scale puts them to either side of it.)"""
    s, a = np.broadcast_to(s, n.shape), np.abs(n)
    low = O.round_to(np.maximum(a - n_error, 0.0) / s * (1.0 - 4.0 * U32), "e4m3")
    high = O.round_to((a + n_error) / s * (1.0 + 4.0 * U32), "e4m3")
    good = (low <= np.abs(q)) & (np.abs(q) <= high) & ((q * n >= 0.0) | (a <= n_error))
    worst = int(np.argmin(good))
    assert good.all(), f"{what}: element {worst}: {q.flat[worst]!r}, between {low.flat[worst]!r} and {high.flat[worst]!r} expected"
