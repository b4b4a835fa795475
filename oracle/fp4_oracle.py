"""Float64 oracle of the 4-bit cache (numpy on the host; definitions only): what
codes and scales stand for, and what a group of values becomes.

32 consecutive values share 2^(s - 127); a code's low three bits are a level, its
high bit the sign; s = 255 makes the group NaN."""
from __future__ import annotations

import numpy as np

from oracle.ssn_oracle import f64 as widen

GROUP = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def unpack(codes):
    """Codes of single elements: the low half of a byte is the first."""
    c = np.asarray(codes)
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], 2 * c.shape[-1])


def pack(c):
    c = np.asarray(c, np.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def values(codes, scales):
    """[.., D] float64 of codes [.., D / 2] and scales [.., D / 32]."""
    c = unpack(codes)
    s = np.repeat(np.asarray(scales).astype(np.int64), GROUP, -1)
    x = np.ldexp(np.where(c > 7, -1.0, 1.0) * LEVELS[c & 7], s - 127)
    return np.where(s == 255, np.nan, x)


def scale_bytes(top):
    """Of the largest magnitudes of groups: the smallest e in -126 .. 125 with
    top < 7 2^e, plus 127; 255 where top is not finite."""
    top = np.asarray(top, np.float64)
    e = np.full(top.shape, -126, np.int64)
    for n in range(-126, 125):
        e[top >= 7.0 * 2.0 ** n] = n + 1
    return np.where(np.isfinite(top), e + 127, 255).astype(np.uint8)


def nearest(v):
    """Level numbers of magnitudes: the nearest one, of two the even one; the
    largest from 5 on."""
    v = np.asarray(v, np.float64)[..., None]
    d = np.abs(v - LEVELS)
    best = d.min(-1, keepdims=True)
    even = np.where(d == best, np.arange(8) % 2, 2)
    return even.argmin(-1)


def group_tops(x):
    x = np.asarray(x)
    return np.abs(x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)).max(-1)


def quantise(x):
    """(codes [.., D / 2], scales [.., D / 32]) of stored values x [.., D]."""
    x = widen(x)
    with np.errstate(invalid="ignore"):
        s = scale_bytes(group_tops(x))
    e = np.repeat(s.astype(np.int64) - 127, GROUP, -1)
    bad = np.repeat(s == 255, GROUP, -1)
    v = np.where(bad, 0.0, x)
    c = nearest(np.abs(np.ldexp(v, np.where(bad, 0, -e)))) + 8 * np.signbit(v)
    return pack(np.where(bad, 0, c)), s
