"""64-bit counterparts of the rotary positions' calls, on numpy arrays: pairs as complex numbers.  Nothing here is shared with
the library."""
from __future__ import annotations

import math

import numpy as np


def frequencies(dim, base=10000.0, scale=1.0, original=None, turns=(1.0, 32.0), divisors=None):
    out = []
    for i in range(dim // 2):
        f = base ** (-2.0 * i / dim)
        if original is None:
            f /= scale
        else:
            r = original * f / (2.0 * math.pi)  # turns over the original length
            keep = 0.0 if r <= turns[0] else 1.0 if r >= turns[1] else (r - turns[0]) / (turns[1] - turns[0])
            f = keep * f + (1.0 - keep) * f / scale
        out.append(f / divisors[i] if divisors is not None else f)
    return np.array(out)


def rotate(x, freq, positions, interleaved=False, magnitude=1.0, inverse=False):
    """x [T][H][D] float64."""
    x = np.array(x, np.float64)
    P = len(freq)
    first = slice(0, 2 * P, 2) if interleaved else slice(0, P)
    second = slice(1, 2 * P, 2) if interleaved else slice(P, 2 * P)
    a = np.outer(np.asarray(positions, np.float64), freq)[:, None, :]
    with np.errstate(invalid="ignore"):
        u, v = x[:, :, first].copy(), x[:, :, second].copy()
        c, s = np.cos(a), -np.sin(a) if inverse else np.sin(a)
        x[:, :, first], x[:, :, second] = magnitude * (u * c - v * s), magnitude * (u * s + v * c)
    return x


def slack(x, freq, positions, interleaved=False, magnitude=1.0):
    """m (|u| + |v|) of each element's pair, and that times its angle (0 outside the turned part): what a rounding of the
    angle's cosine and sine, and one of the angle itself, are relative to."""
    x = np.abs(np.asarray(x, np.float64))
    P = len(freq)
    first = slice(0, 2 * P, 2) if interleaved else slice(0, P)
    second = slice(1, 2 * P, 2) if interleaved else slice(P, 2 * P)
    both = magnitude * (x[:, :, first] + x[:, :, second])
    a = np.abs(np.outer(np.asarray(positions, np.float64), freq))[:, None, :]
    near, far = np.zeros_like(x), np.zeros_like(x)
    near[:, :, first] = near[:, :, second] = both
    far[:, :, first] = far[:, :, second] = both * a
    return near, far


def bound(magnitude):
    """What the largest magnitude of a turned part is multiplied by, in fp32."""
    return np.float32(math.sqrt(2.0) * float(np.float32(magnitude)))


def key_limit(key, pairs, magnitude):
    """[T][H]: what an appended key's exponent goes by."""
    mags = np.where(np.isfinite(key), np.abs(key), 0.0)
    turned = (mags[:, :, :2 * pairs].max(axis=2).astype(np.float32) * bound(magnitude)).astype(np.float64)
    turned = np.minimum(turned, float(np.finfo(np.float32).max))
    if 2 * pairs < key.shape[2]:
        turned = np.maximum(turned, mags[:, :, 2 * pairs:].max(axis=2))
    return turned
