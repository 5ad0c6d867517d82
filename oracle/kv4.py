"""The 4-bit row format of the cache, from its definition, on the CPU.

A row of 128 values is four groups of 32; a group keeps lo = min(x), s = bf16((max(x) - lo) / 15)
and c = round_half_even((x - lo) / s); x stands for lo + s * c.  Differences and quotients are
IEEE single precision, as the definition says, so codes can be compared for equality; a scale
below 2^-100 is kept as 0.
"""
import numpy as np

GROUP = 32


def round_bf16(x):
    """Single-precision numbers rounded to bf16 (ties to even), as single precision."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def quantise(x):
    """x: [..., 128] numbers that are bf16.  Returns (codes, s, lo), the last two [..., 4]."""
    x = np.asarray(x, dtype=np.float32).reshape(*np.shape(x)[:-1], 4, GROUP)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        rng = hi - lo
        s = round_bf16(rng / np.float32(15))
        s = np.where(s >= np.float32(2.0 ** -100), s, np.float32(0))
        safe = np.where(s > 0, s, np.float32(1))[..., None]
        c = np.where(s[..., None] > 0, np.rint((x - lo[..., None]) / safe), 0)
    bad = ~np.isfinite(rng)
    s, lo = np.where(bad, np.nan, s), np.where(bad, np.nan, lo)
    c = np.where(bad[..., None], 0, c)
    assert c.min() >= 0 and c.max() <= 15
    return c.astype(np.int64), s.astype(np.float64), lo.astype(np.float64)


def values(codes, s, lo):
    """What the codes stand for, in double precision, [..., 128]."""
    v = lo[..., None] + s[..., None] * codes
    return v.reshape(*v.shape[:-2], 4 * GROUP)


def spread(codes, s):
    """s c: the part of a value that the attention weights multiply after rounding."""
    v = s[..., None] * codes
    return v.reshape(*v.shape[:-2], 4 * GROUP)
