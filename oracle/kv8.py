"""The 8-bit paged cache's values, blocks and selection (test infrastructure
only, like the rest of oracle/), written from the definitions in include/hh.h.
Attention over its values is ``kv4.attend``, rotation ``kv4.rotate``.

A block's keys (and its values) have one scale 2^e, e the least integer from
-20 to 9 with max|x| <= 127 * 2^e; codes are clamp(rint(x / 2^e), -127, 127).
"""
from __future__ import annotations

import math

import numpy as np

PAGE, HEAD, BLOCK = 16, 64, 2176
LOW, HIGH = -20, 9


def exponent(top: float) -> int:
    for e in range(LOW, HIGH):
        if top <= 127 * 2.0 ** e:
            return e
    return HIGH


class Block:
    """One (page, kv head): codes [2][16, 64], exponents, marks, for keys and values."""

    def __init__(self):
        self.codes = [np.zeros((PAGE, HEAD), np.int64) for _ in "kv"]
        self.exp = [LOW, LOW]
        self.bad = [np.zeros(PAGE, bool) for _ in "kv"]

    def put(self, slot: int, k: np.ndarray, v: np.ndarray) -> None:
        """One call's rows [n, 64] (finite or not) at slots slot .. slot + n - 1."""
        for i, x in enumerate((k, v)):
            x = np.asarray(x, dtype=np.float64)
            bad = ~np.isfinite(x).all(-1)
            x = np.where(bad[:, None], 0.0, x)
            e = exponent(float(np.abs(x).max(initial=0.0)))
            if slot > 0:
                e = max(e, self.exp[i])
            c = np.zeros((PAGE, HEAD), np.int64)
            c[:slot] = np.rint(self.codes[i][:slot] * 2.0 ** (self.exp[i] - e)) if slot else 0
            c[slot:slot + len(x)] = np.clip(np.rint(x * 2.0 ** -e), -127, 127)
            mark = np.zeros(PAGE, bool)
            mark[:slot] = self.bad[i][:slot]
            mark[slot:slot + len(x)] = bad
            self.codes[i], self.exp[i], self.bad[i] = c, e, mark

    def values(self):
        return tuple(np.where(b[:, None], np.nan, c * 2.0 ** e) for c, e, b in zip(self.codes, self.exp, self.bad))

    def summary(self):
        """(whole numbers m, scale of the mean key)."""
        total = self.codes[0].sum(0)
        j = 0
        while np.abs(total).max() > 127 * 2 ** j:
            j += 1
        return np.rint(total / 2.0 ** j).astype(np.int64), 2.0 ** (self.exp[0] + j - 4)

    def bytes(self) -> np.ndarray:
        """The defined bytes, 0 .. 2127."""
        out = np.zeros(2128, np.uint8)
        for slot in range(PAGE):
            for d in range(HEAD):
                h, g, j = d // 32, d % 32 // 8, d % 8
                out[256 * g + 16 * slot + 8 * h + j] = self.codes[0][slot, d] + 128
                g, i, r, j = slot // 4, slot % 4, d // 4, d % 4
                out[1024 + 256 * g + 16 * r + 4 * j + i] = self.codes[1][slot, d] + 128
        m, s = self.summary()
        out[2048:2112] = m.astype(np.int8).view(np.uint8)
        half = out[2112:].view(np.float16)
        half[0], half[1], half[4] = 2.0 ** self.exp[0], 2.0 ** self.exp[1], s
        for i in range(2):
            out[2116:2120].view(np.uint16)[i] = sum(int(b) << n for n, b in enumerate(self.bad[i]))
        return out


class Cache:
    """Sequences of blocks [sequence][page][head], appended to as hh_kv8_append does."""

    def __init__(self, seqs: int, pages: int, heads: int):
        self.blocks = [[[Block() for _ in range(heads)] for _ in range(pages)] for _ in range(seqs)]
        self.heads, self.pages = heads, pages

    def append(self, seq: int, first: int, k: np.ndarray, v: np.ndarray) -> None:
        """fp32 rows [n, heads, 64] (keys rotated) at positions first, ..."""
        n, pos = len(k), max(first, 0)
        end = min(first + n, self.pages * PAGE)
        while pos < end:
            page, stop = pos // PAGE, min((pos // PAGE + 1) * PAGE, end)
            for h in range(self.heads):
                at = slice(pos - first, stop - first)
                self.blocks[seq][page][h].put(pos % PAGE, k[at, h], v[at, h])
            pos = stop

    def values(self, seq: int, n: int):
        """fp64 keys and values [n, heads, 64] of the first n positions."""
        out = [np.zeros((self.pages * PAGE, self.heads, HEAD)) for _ in "kv"]
        for p, page in enumerate(self.blocks[seq]):
            for h, b in enumerate(page):
                for x, y in zip(out, b.values()):
                    x[p * PAGE:(p + 1) * PAGE, h] = y
        return out[0][:n], out[1][:n]


def query_codes(q: np.ndarray) -> np.ndarray:
    """Whole numbers [64] of a group's queries [G, 64] (rotated, fp64)."""
    total = np.zeros(HEAD)
    for x in np.asarray(q, dtype=np.float64):
        total = total + x
    top = np.abs(total).max()
    if not np.isfinite(total).all() or top == 0:
        return np.zeros(HEAD, np.int64)
    f = math.ceil(math.log2(top / 127))
    while top > 127 * 2.0 ** f:
        f += 1
    while top <= 127 * 2.0 ** (f - 1):
        f -= 1
    return np.rint(total / 2.0 ** f).astype(np.int64)


def select(q: np.ndarray, blocks, pos: int, n: int, first: int, last: int) -> np.ndarray:
    """The n blocks of a row at `pos` for the queries [G, 64] of a kv head, whose
    blocks are blocks[page]; -1 behind the last."""
    out = np.full(n, -1, np.int64)
    count = min(pos // PAGE + 1, len(blocks)) if pos >= 0 else 0
    if count <= n:
        out[:count] = np.arange(count)
        return out
    a = query_codes(q)
    score = []
    for b in range(first, count - last):
        m, s = blocks[b].summary()
        score.append((-float(int(a @ m)) * s, b))
    best = [b for _, b in sorted(score)[:n - first - last]]
    out[:] = sorted(list(range(first)) + best + list(range(count - last, count)))
    return out
