"""How far an attention output may be from the exact one when its weights are rounded to bf16 each for the product with V: a bound that a single
value row in the wrong place exceeds."""

import numpy as np

from tests import continuation_oracle as orc


def attend(q, k, v, scale):
    """One row and KV head in 64 bits: q [G, D], k and v [n, D] -> (out, weights [G, n])."""
    s = q @ k.T * scale
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, p


def delta(p, v):
    """Each weight is rounded to 8 significant bits: by half a unit of the last, at most 2^-8 of it, either way, and the weights of unrelated keys
    independently of each other: their standard deviation is 2^-8 / sqrt(3) of the weight at most (that of an even spread over the unit),
    that of the output sqrt(sum w^2 v^2) times as much.  Six of those (chance 2e-9), and what sums and exponentials in fp32 add (2e-5 of sum w |v|)."""
    return 6 * 2.0 ** -8 / np.sqrt(3) * np.sqrt(p ** 2 @ v ** 2) + 2e-5 * (p @ np.abs(v)) + 1e-30


def check(got, q, k, v, scale):
    """Where got is the bf16 rounding of a number within delta of the exact output."""
    want, p = attend(q, k, v, scale)
    return orc.rounded_within(got, want, delta(p, v))
