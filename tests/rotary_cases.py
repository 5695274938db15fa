"""Bounds of rotations and of what is stored of them in 8 bits, and cases of appends."""
import numpy as np

BITS = {"f16": 11, "bf16": 8}  # of a rounding: half a step is 2^-bits of the value
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half a step of the smallest values


def turned_bound(x, magnitude):
    """How far a turned element, before its last rounding, may be off what float64 gives.  a c - b s in float: c and s are off
    by 2^-24 of themselves (they are at most the magnitude), and 2^-50 of it as the angles and their cosines are in double in
    another order; each product is rounded, and their difference: (2 * 2^-24) (|a| + |b|) magnitude and 2^-24 of the result,
    which is at most that size: three times 2^-24, and 5% for terms of higher order."""
    return 1.05 * 3 * 2.0 ** -24 * magnitude * x


def pair_size(x, pairs, interleaved):
    """|a| + |b| of every element's pair; of the elements that stay, 0."""
    s = np.zeros_like(x)
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    s[..., a] = s[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return s


def rotate_bound(x, want, pairs, interleaved, magnitude, kind):
    """... and the rounding to 16 bits."""
    off = turned_bound(pair_size(x, pairs, interleaved), magnitude)
    return off + 2.0 ** -BITS[kind] * (np.abs(want) + off) + TINY[kind]
