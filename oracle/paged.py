"""O10: rotary positions scaled for long contexts, and a paged cache in 8 bits with a scale for each page and head.

Rotations of angles p f_i in fp64 for what is compared within a tolerance; codes are defined by fp32 arithmetic (each
product and sum rounded), which numpy float32 arrays evaluate exactly, so they are compared bit for bit.
"""
from __future__ import annotations

import math

import numpy as np

E_MIN, E_MAX = -100, 120
TOP = {"e4m3": 448.0, "int8": 127.0}


def frequencies(rot, theta=10000.0, scaling="plain", factor=1.0, low=1.0, high=4.0, context=0):
    """Radians a position of the rot / 2 pairs, one pair at a time."""
    out = []
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            turns = context * f / (2.0 * math.pi)
            keep = min(max((turns - low) / (high - low), 0.0), 1.0)
            f = keep * f + (1.0 - keep) * f / factor
        elif scaling == "ramp":
            def pair(turns):
                return rot * math.log(context / (2.0 * math.pi * turns)) / (2.0 * math.log(theta))
            a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
            slow = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = (1.0 - slow) * f + slow * f / factor
        out.append(f)
    return np.array(out)


def table(positions, freq, magnitude=1.0):
    """(cos, sin) [n][pairs][2] in fp64."""
    a = np.asarray(positions, dtype=np.float64)[:, None] * freq[None, :]
    return magnitude * np.stack([np.cos(a), np.sin(a)], -1)


def rotate(x, cs, layout):
    """x [n, heads, D] by cs [n, pairs, 2], in the type that both have."""
    r = 2 * cs.shape[1]
    i0 = np.arange(r // 2) if layout == "half" else np.arange(0, r, 2)
    i1 = i0 + r // 2 if layout == "half" else i0 + 1
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    y = x.copy()
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i1] * c + x[..., i0] * s
    return y


def _e4m3_values():
    v = np.zeros(256)
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        x = m / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
        v[code] = -x if code & 128 else x
    return v


E4M3 = _e4m3_values()          # (of the two NaN codes: what their bits would be)


def decode(codes, fmt):
    """Codes (uint8 for e4m3, int8) as numbers, fp64."""
    return E4M3[codes] if fmt == "e4m3" else codes.astype(np.float64)


def encode(x, fmt):
    """fp32 numbers to codes: nearest, ties to even, the largest beyond the range; NaN is zero."""
    x = np.where(np.isnan(x), 0.0, x.astype(np.float64))
    if fmt == "int8":
        return np.clip(np.rint(x), -127, 127).astype(np.int8)
    mag = np.minimum(np.abs(x), 448.0)
    v = E4M3[:127]
    hi = np.clip(np.searchsorted(v, mag, side="left"), 1, 126)
    lo = hi - 1
    mid = (v[lo] + v[hi]) / 2
    up = (mag > mid) | ((mag == mid) & (hi % 2 == 0))
    return (np.where(up, hi, lo) + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def least_scale(most, fmt):
    """2^e, e the least integer with most <= top 2^e."""
    e = E_MIN
    while e < E_MAX and float(most) > TOP[fmt] * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def append_page(codes, scale, held, new, fmt):
    """One head's page: codes [page, D] (changed in place), its scale, the tokens it holds, new rows [m, D] fp32.  The
    scale afterwards."""
    new = np.asarray(new, dtype=np.float32)
    finite = np.where(np.isfinite(new), np.abs(new), np.float32(0))
    most = finite.max()
    if held > 0 and float(most) <= TOP[fmt] * float(scale):
        now = np.float32(scale)
    else:
        now = least_scale(most, fmt)
        if held > 0:
            now = max(now, np.float32(scale))
            with np.errstate(under="ignore"):
                less = np.float32(scale) / now
                codes[:held] = encode(decode(codes[:held], fmt).astype(np.float32) * less, fmt)
    with np.errstate(under="ignore", invalid="ignore"):
        codes[held:held + len(new)] = encode(new / now, fmt)
    return now
