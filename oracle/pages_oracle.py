"""Float64 statement of rotary positions, of a paged cache in 8 bits and of attention over it: one head of one sequence at a time, plain
numpy; shares no code with the GPU path."""
import math

import numpy as np

BLOCK, LOW, TOP = 16, -40, 448.0


def frequencies(dim, base, scaling=None, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    """(radians a position of every pair, amplitude)."""
    if scaling == "base":
        base = base * factor ** (dim / (dim - 2))
    f = np.array([base ** (-2.0 * c / dim) for c in range(dim // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        part = np.clip((original * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
    elif scaling == "ramp":
        def pair(turns):
            return dim * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(pair(fast))), min(dim - 1, math.ceil(pair(slow)))
        part = 1 - np.clip((np.arange(dim // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
    else:
        return f, 1.0
    f = part * f + (1 - part) * f / factor
    return f, 0.1 * math.log(factor) + 1 if scaling == "ramp" and factor > 1 else 1.0


def pairs(dim, interleaved):
    c = np.arange(dim // 2)
    return (2 * c, 2 * c + 1) if interleaved else (c, c + dim // 2)


def rotate(x, positions, f, amplitude=1.0, interleaved=False, inverse=False):
    """x [tokens, d] (or [tokens, heads, d]) at positions [tokens]."""
    x = np.asarray(x, dtype=np.float64)
    # (whole turns go first, in integers as far as they are: the angle of a far position in 64 bits)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * f
    if inverse:
        angle = -angle
    a, b = pairs(2 * len(f), interleaved)
    cos, sin = amplitude * np.cos(angle), amplitude * np.sin(angle)
    if x.ndim == 3:
        cos, sin = cos[:, None], sin[:, None]
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _all_codes():
    v = np.empty(256)
    for i in range(256):
        s, e, m = i >> 7, i >> 3 & 15, i & 7
        v[i] = math.nan if (i & 127) == 127 else (m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if s else 1)
    return v


CODES = _all_codes()
_POSITIVE = CODES[:127]                                     # ascending


def code_of(x):
    """e4m3 codes of values within 448: to nearest, ties to the even code; what is not finite becomes NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    c = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(np.signbit(x), c + 128, c)
    return np.where(np.isfinite(x), c, 127).astype(np.uint8)


def exponent(top):
    """Of the smallest power of two, from 2^-40 on, with which top stays within 448 of it."""
    e = LOW
    while top > TOP * 2.0 ** e:
        e += 1
    return e


def values(codes, exponents):
    """[slots, d] of codes [slots, d] and the exponents of 16 slots each."""
    return CODES[codes] * 2.0 ** np.repeat(np.asarray(exponents, dtype=np.float64), BLOCK)[:len(codes), None]


def append(codes, exponents, n, rows):
    """One head's codes [slots, d] and exponents [slots / 16] after rows [new, d] were written behind the first n."""
    codes, exponents = codes.copy(), list(exponents)
    for lo in range(n // BLOCK * BLOCK, n + len(rows), BLOCK):
        a, z = max(lo, n), min(lo + BLOCK, n + len(rows))
        if a >= z:
            continue
        new = rows[a - n:z - n]
        e = exponent(np.abs(new[np.isfinite(new)]).max(initial=0.0))
        if a > lo:
            had = exponents[lo // BLOCK]
            if e > had:
                old = CODES[codes[lo:a]]
                codes[lo:a] = np.where(np.isnan(old), codes[lo:a], code_of(old * 2.0 ** (had - e)))
            e = max(e, had)
        codes[a:z] = code_of(new * 2.0 ** -e)
        exponents[lo // BLOCK] = e
    return codes, exponents


def attend(q, k, v, n, scale, softcap=0.0):
    """q [new, G, d] over k, v [n + new, d]: out [new, G, d], lse [new, G], and the probabilities [new, G, n + new]."""
    t, g, d = q.shape
    out, lse, p = np.zeros((t, g, d)), np.full((t, g), -np.inf), np.zeros((t, g, len(k)))
    for i in range(t):
        x = (q[i] @ k[:n + i + 1].T) * scale
        if softcap:
            x = softcap * np.tanh(x / softcap)
        top = x.max(axis=1, keepdims=True)
        e = np.exp(x - top)
        lse[i] = top[:, 0] + np.log(e.sum(axis=1))
        e /= e.sum(axis=1, keepdims=True)
        out[i] = e @ v[:n + i + 1]
        p[i, :, :n + i + 1] = e
    return out, lse, p
