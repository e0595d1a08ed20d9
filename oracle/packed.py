"""fp64 oracle of caches held in 4 bits (test infrastructure only): the codes of a
group, the bytes of a row and the values they stand for.

Plain NumPy, written from the definitions; it shares nothing with the HIP path.
"""
from __future__ import annotations

import numpy as np

GROUP = 32


def row_bytes(d):
    return 5 * d // 4


def quantise(x):
    """x [..., d] (exact in float32): codes [..., d], scales and bases [..., d / 32] (float16)."""
    x = np.asarray(x, np.float32)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    whole = np.isfinite(g).all(-1)
    g = np.clip(np.where(whole[..., None], g, 0), np.float32(-16384), np.float32(16384))
    m, M = g.min(-1), g.max(-1)
    s = ((M - m) / np.float32(15)).astype(np.float16)
    b = (m - np.float32(16) * s.astype(np.float32)).astype(np.float16) + np.float16(0)       # + 0: no negative zero
    t = (g - b.astype(np.float32)[..., None]).astype(np.float64)
    n = np.zeros(g.shape, np.int64)
    for k in range(1, 16):                            # the largest k whose border does not lie above t
        n[(t >= (15.5 + k) * s.astype(np.float64)[..., None]) & (s > 0)[..., None]] = k
    return n.reshape(x.shape), s, np.where(whole, b, np.float16(np.nan))


def quantise_group(x):
    """One group of 32 numbers: codes, scale and base."""
    n, s, b = quantise(x)
    return n, s[0], b[0]


def values(n, s, b):
    """What codes stand for: s (16 + n) + b, rounded once to fp16 (as float64)."""
    s, b = (np.repeat(np.asarray(x, np.float64), GROUP, -1) for x in (s, b))
    with np.errstate(over="ignore", invalid="ignore"):
        return (s * (16 + np.asarray(n)) + b).astype(np.float16).astype(np.float64)


def pack(k, v):
    """Rows [..., 5 d / 4] (uint8) of keys and values [..., d]."""
    k, v = np.asarray(k, np.float32), np.asarray(v, np.float32)
    d, lead = k.shape[-1], k.shape[:-1]
    out = np.zeros((int(np.prod(lead, dtype=np.int64)), row_bytes(d)), np.uint8)
    for at, par, x in ((0, d, k), (d // 2, d + d // 8, v)):
        n, s, b = quantise(x.reshape(out.shape[0], d))
        for w in range(d):
            bit = 32 * (w // 8) + 16 * (w % 2) + 4 * (w % 8 // 2)
            out[:, at + bit // 8] |= (n[:, w] << bit % 8).astype(np.uint8)
        sb = np.stack([s, b], -1).astype("<f2")
        out[:, par:par + d // 8] = np.ascontiguousarray(sb).view(np.uint8).reshape(out.shape[0], d // 8)
    return out.reshape(*lead, row_bytes(d))


def unpack(rows):
    """Keys and values [..., d] (float64) that rows stand for."""
    rows = np.asarray(rows, np.uint8)
    d, flat = rows.shape[-1] * 4 // 5, rows.reshape(int(np.prod(rows.shape[:-1])), rows.shape[-1])
    res = []
    for at, par in ((0, d), (d // 2, d + d // 8)):
        n = np.zeros((flat.shape[0], d), np.int64)
        for w in range(d):
            bit = 32 * (w // 8) + 16 * (w % 2) + 4 * (w % 8 // 2)
            n[:, w] = flat[:, at + bit // 8] >> bit % 8 & 15
        sb = np.ascontiguousarray(flat[:, par:par + d // 8]).view("<f2").reshape(flat.shape[0], d // GROUP, 2)
        res.append(values(n, sb[..., 0], sb[..., 1]).reshape(*rows.shape[:-1], d))
    return res
