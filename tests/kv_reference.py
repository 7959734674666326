"""Plain 64-bit definitions of the KV cache's operators (numpy, on the CPU): rotary
positions, block quantisation, and attention with an explicit visibility mask.
Written from the formulas; slow and small."""
from __future__ import annotations

import math

import numpy as np

LARGEST = {"fp8": 448.0, "fp4": 6.0}
MIN_EXP = -110


def e4m3_values():
    """Value of every e4m3 code (two of them NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.ldexp(1 + m / 8, e - 7) if e else math.ldexp(m / 8, -6)
        if e == 15 and m == 7:
            v = math.nan
        out[c] = -v if c & 128 else v
    return out


def e2m1_values():
    v = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return np.array(v + [-x for x in v])


def values_of(fmt):
    return e4m3_values() if fmt == "fp8" else e2m1_values()


def nearest_code(y, fmt):
    """Code whose value is nearest to each y, ties to the even code; the sign bit is y's."""
    half = 128 if fmt == "fp8" else 8
    levels = values_of(fmt)[:half]
    if fmt == "fp8":
        levels = levels[:127]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(levels, a), 1, len(levels) - 1)
    lo = hi - 1
    dl, dh = a - levels[lo], levels[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (pick + np.where(np.signbit(y), half, 0)).astype(np.uint8)


def quantise(x, fmt):
    """(codes [..., dim], scale bytes [..., dim / 32]) of rows in 64 bits; codes one a byte."""
    b = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(b).all(-1)
    amax = np.where(bad, 0.0, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1))
    k = np.full(amax.shape, MIN_EXP)
    for at in np.ndindex(amax.shape):
        e = MIN_EXP
        if amax[at] > 0:
            e = max(MIN_EXP, math.frexp(amax[at])[1] - 12)
        while amax[at] > math.ldexp(LARGEST[fmt], e):
            e += 1
        k[at] = e
    y = np.ldexp(np.where(bad[..., None], 0.0, b), -k[..., None])
    codes = nearest_code(y, fmt).reshape(x.shape)
    return codes, np.where(bad, 255, k + 127).astype(np.uint8)


def dequantise(codes, scale, fmt):
    s = np.where(scale == 255, math.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return values_of(fmt)[codes] * np.repeat(s, 32, axis=-1)


def pack(codes, fmt):
    """The bytes of a row: e2m1 codes two a byte, the even element in the low half."""
    return codes if fmt == "fp8" else (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(rows, fmt):
    if fmt == "fp8":
        return rows
    return np.stack([rows & 15, rows >> 4], -1).reshape(rows.shape[:-1] + (-1,))


def rotate(x, cos, sin, interleaved, adjoint=False, dtype=np.float64):
    """x [tokens, heads, dim], cos and sin [tokens, rot / 2]; every product and sum
    rounded to ``dtype``."""
    x = x.astype(dtype)
    c, s = cos.astype(dtype)[:, None], sin.astype(dtype)[:, None]
    if adjoint:
        s = -s
    half = cos.shape[-1]
    i = np.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = x[..., ia], x[..., ib]
    y = x.copy()
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def frequencies(rot, theta, kind="plain", factor=1.0, low=1.0, high=32.0, trained=0.0):
    out = []
    base = theta * factor ** (rot / (rot - 2)) if kind == "base" else theta
    for i in range(rot // 2):
        w = base ** (-2.0 * i / rot)
        turns = trained * w / (2 * math.pi)
        if kind == "linear":
            w = w / factor
        elif kind == "turns":
            g = min(max((turns - low) / (high - low), 0.0), 1.0)
            w = g * w + (1 - g) * w / factor
        elif kind == "index":
            def where(n):
                return rot * math.log(trained / (n * 2 * math.pi)) / (2 * math.log(theta))
            a = min(max(math.floor(where(high)), 0), rot - 1)
            b = min(max(math.ceil(where(low)), 0), rot - 1)
            b = b if b > a else a + 0.001
            g = 1 - min(max((i - a) / (b - a), 0.0), 1.0)
            w = g * w + (1 - g) * w / factor
        out.append(w)
    return np.array(out)


def attention(q, k, v, seen, scale):
    """q [rows, dim], k and v [tokens, dim], seen [rows, tokens]: (out, lse, slack) in 64
    bits.  slack [rows, dim] is sum_j w_j |v_j|, what rounding errors of the
    weights scale with; hidden tokens never enter."""
    rows, dim = q.shape
    out, lse = np.zeros((rows, dim)), np.full(rows, -np.inf)
    slack, spread = np.zeros((rows, dim)), np.zeros(rows)
    for r in range(rows):
        at = np.flatnonzero(seen[r])
        if not len(at):
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = scale * (k[at] @ q[r])
            top = s.max()
            p = np.exp(s - top)
            total = p.sum()
            out[r] = (p / total) @ v[at]
            slack[r] = (p / total) @ np.abs(v[at])
            lse[r] = -np.inf if total == 0 else top + np.log(total)
            spread[r] = (abs(scale) * (np.abs(k[at]) @ np.abs(q[r]))).max()
    return out, lse, slack, spread
