"""Bounds of a serving step's parts, each against float64 on what that part was given: queries and keys against the rotation of
the step's vectors, attention against the softmax over what the cache holds."""
import numpy as np

import rotary_cases as B
from oracle import kv_cache as kv


def key_bound(x, want, pairs, scale):
    """A key as the cache holds it, against float64's: the rotation in float, half a step of 8 bits (2^-4 of the value), or half a
    smallest step (2^-10 of the scale) once when stored and, in all, no more than once again for each time that the scale
    doubled later, which adds up to less than another one of the scale that there is now."""
    off = B.turned_bound(B.pair_size(x, pairs, False), 1.0)
    return off + 2.0 ** -4 * (np.abs(want) + off) + 2 * 2.0 ** -10 * scale


def attention_bound(ref, keys, dim, top):
    """One step's attention, bfloat16 results, weights to 11 bits; `top`: the largest |value| that a row sees.  Scales are powers of
    two, whose logarithms are exact."""
    return kv.attention_bound(*ref, keys, dim, 8, 11, top)
