"""The 4-bit paged cache's values, blocks and attention (test infrastructure
only, like the rest of oracle/), written from the definitions in include/hh.h.

Key and value rows are held in groups of 32 of a head's 64 dimensions: scale
s = max|x| / 7 in fp32, rounded to 8 significant bits and to a multiple of
2^-24, at most 2720; code c = clamp(rint(x / s), -7, 7) with the division in
fp32; value c * s.  A row with an infinity or NaN has NaN scales.
"""
from __future__ import annotations

import numpy as np

PAGE, HEAD, BLOCK = 16, 64, 1152


def quantize(x: np.ndarray):
    """Codes int [..., 64] and scales float64 [..., 2] of rows [..., 64]."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        g = x.reshape(*x.shape[:-1], 2, 32)
        t = np.max(np.abs(g), axis=-1) / np.float32(7.0)
        _, e = np.frexp(t.astype(np.float64))
        step = np.exp2(np.maximum(e - 8, -24).astype(np.float64))
        s = np.minimum(np.rint(t / step) * step, 2720.0)
        bad = ~np.isfinite(x).all(axis=-1)
        s = np.where(bad[..., None], np.nan, s)
        r = g / s[..., None].astype(np.float32)
        c = np.where(s[..., None] > 0, np.clip(np.rint(r), -7, 7), 0.0)
        return np.nan_to_num(c).astype(np.int64).reshape(x.shape), s


def dequantize(c: np.ndarray, s: np.ndarray) -> np.ndarray:
    """fp64 values c * s."""
    return (c.reshape(*c.shape[:-1], 2, 32) * s[..., None]).reshape(c.shape)


def values(x: np.ndarray) -> np.ndarray:
    """The fp64 values that rows [..., 64] are held as."""
    return dequantize(*quantize(x))


def put(block: np.ndarray, slot: int, k: np.ndarray, v: np.ndarray) -> None:
    """Write one key row and one value row into a slot of a block (uint8 [1152])."""
    words, scales = block[:1024].view(np.uint16), block[1024:].view(np.float16)
    kc, ks = quantize(k)
    vc, vs = quantize(v)
    for d in range(HEAD):
        t, g, e = d // 32, d % 32 // 8, d % 8
        w, j = 4 * (16 * g + slot) + 2 * t + e % 2, e // 2
        words[w] = (int(words[w]) & ~(15 << 4 * j)) | (int(kc[d]) + 8) << 4 * j
        w, j = 256 + 4 * (16 * (slot // 4) + d // 4) + slot % 4, d % 4
        words[w] = (int(words[w]) & ~(15 << 4 * j)) | (int(vc[d]) + 8) << 4 * j
    for t in range(2):
        scales[2 * slot + t] = ks[t]
        scales[32 + 16 * t + slot] = vs[t]


def rotate(x: np.ndarray, table: np.ndarray, pos: np.ndarray) -> np.ndarray:
    """Rows x [n, heads, 64] rotated by the fp32 (cos, sin) of their positions
    in a table [len, 32, 2], in fp64."""
    x = np.asarray(x, dtype=np.float64)
    c, s = (table[pos, :, i].astype(np.float64)[:, None] for i in (0, 1))
    a, b = x[..., :32], x[..., 32:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float, first: int) -> np.ndarray:
    """Rows q [n, heads, 64] at positions first, first + 1, ... over keys and
    values [T, kv heads, 64] of positions 0 .. T - 1, fp64; rows with nothing to
    attend to are 0."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    group = q.shape[1] // k.shape[1]
    out = np.zeros_like(q)
    with np.errstate(invalid="ignore"):
        for i in range(q.shape[0]):
            n = min(first + i + 1, k.shape[0])
            if n <= 0:
                continue
            for h in range(q.shape[1]):
                s = k[:n, h // group] @ q[i, h] * scale
                w = np.exp(s - s.max())
                out[i, h] = w @ v[:n, h // group] / w.sum()
    return out
