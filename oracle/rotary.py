"""Rotations by position and appends to a block cache whose scales follow what
its blocks hold, written from their definitions, token by token, in float64
(the scales' arithmetic in float32 where the operator's is)."""
import math

import numpy as np

from oracle.kv_cache import round_e4m3

LEAST, MOST = -64, 64  # exponents of the scales


def frequencies(dim, base=10000.0, scaling=None, factor=1.0, length=0.0, low=1.0, high=32.0):
    """(frequencies of the dim / 2 pairs, magnitude), pair by pair."""
    if scaling == "base":
        base = base * factor ** (dim / (dim - 2))
    freqs = []
    for i in range(dim // 2):
        f = base ** (-2.0 * i / dim)
        if scaling == "linear":
            f /= factor
        elif scaling == "ramp":
            # Pair numbers (real) at which `turns` turns fit the length; whole pairs around them.
            at = lambda turns: dim * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
            first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), dim - 1)
            slow = min(max((i - first) / (last - first if last > first else 0.001), 0.0), 1.0)
            f = (1 - slow) * f + slow * f / factor
        elif scaling == "bands":
            turns = length * f / (2 * math.pi)
            if turns < low:
                f /= factor
            elif turns <= high:
                keep = (turns - low) / (high - low)
                f = keep * f + (1 - keep) * f / factor
        freqs.append(f)
    return np.array(freqs), 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0


def rotate(x, positions, freqs, magnitude=1.0, interleaved=False, reverse=False):
    """x (tokens, heads, dim), its first 2 len(freqs) elements turned as complex numbers."""
    y = np.array(x, dtype=np.float64)
    n = len(freqs)
    for t, p in enumerate(positions):
        turn = magnitude * np.exp((-1j if reverse else 1j) * (float(p) * np.asarray(freqs)))
        a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
        with np.errstate(invalid="ignore"):
            re, im = y[t][:, a].copy(), y[t][:, b].copy()
            y[t][:, a] = re * turn.real - im * turn.imag
            y[t][:, b] = im * turn.real + re * turn.imag
    return y


def power_of_two(x):
    """The smallest power of two E, from 2^LEAST to 2^MOST, with x <= 448 E."""
    e = LEAST
    while e < MOST and x > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append_scaled(x, slots, codes, scales):
    """One cache (blocks, heads, block_size, dim) of 8-bit numbers ``codes`` and
    its ``scales`` (blocks, heads), float32, with the vectors x (tokens, heads,
    dim) at their slots.  Returns (codes, scales, new): new values as they are
    before their rounding to 8 bits, earlier ones as they are stored."""
    codes, scales = np.array(codes, dtype=np.float64), np.array(scales, dtype=np.float32)
    blocks, heads, bs, _ = codes.shape
    runs = {}
    for t, s in enumerate(slots):
        if 0 <= s < blocks * bs:
            runs.setdefault(int(s) // bs, []).append((t, int(s) % bs))
    fresh = np.zeros((blocks, bs), dtype=bool)
    for b, rows in runs.items():
        begin = rows[0][1]
        for h in range(heads):
            held = np.concatenate([x[t, h] for t, _ in rows])
            held = np.abs(held[np.isfinite(held)])
            need = np.float32(power_of_two(held.max() if held.size else 0.0))
            old = scales[b, h]
            scale = need
            if begin and old > 0 and np.isfinite(old):
                scale = max(old, need)
                if scale > old:
                    by = np.float32(old / scale)
                    earlier = codes[b, h, :begin].astype(np.float32) * by
                    codes[b, h, :begin] = round_e4m3(earlier.astype(np.float64))
            scales[b, h] = scale
            for t, at in rows:
                codes[b, h, at] = x[t, h] / float(scale)
                fresh[b, at] = True
    return codes, scales, fresh
