"""How far the norm of the fp32 feed-forward products' error may be from the result's, for inputs as in the tests (x and dout
of deviation 1, weights of K^-1/2).

A sum of n products that is formed one after another rounds n times, by a deviation of 2^-24 / sqrt(3) of the sum so far (a
value is off by up to half a step, 2^-24 of it).  Terms of either sign make sums that grow with the square root, so the
roundings add up to 2^-24 sqrt(sum of k / 3) = 2^-24 n / sqrt(6), against a result of sqrt(n): 2^-24 sqrt(n / 6).  Sums that
are formed in parts are off by less.  An output has two such sums, and the activation takes an error of the gate times its
slope (1.1 at most) over its own deviation (0.597 of SiLU for a gate of deviation 1): 1 + 1.1 / 0.597 = 2.9 in all; the
gradients of the projections have no more.  The activation itself and its products: 2^-21.  Thousands of outputs keep the norm
within a few percent of its expectation; half as much again is allowed."""
import math

SIZES = [(333, 260, 103), (5, 2048, 1288), (300, 512, 1032), (16, 264, 520), (1030, 520, 2600), (33, 2048, 520), (128, 1031, 260),
         (1, 2056, 1384)]


def bounds(M, K, F):
    """{"out", "dx", "dw"}: bounds of |error| / |result| (2-norms)."""
    sums = lambda n: 2.0 ** -24 * math.sqrt(n / 6)  # noqa: E731
    first = 2.9 * sums(K) + 2.0 ** -21
    return {"out": 1.5 * first, "dx": 1.5 * (first + sums(2 * F)), "dw": 1.5 * (first + sums(M))}


def off(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())
