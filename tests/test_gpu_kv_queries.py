"""Queries that are not finite, on both quantized caches: a row that sees a key gives NaN, in calls of any
size and queries of any type, a row that sees none gives 0, and other rows and heads stay.

Those share a wave with it, whose columns raise their bases together, so that their roundings may be others.
Each result is within e of the exact weights, e = 2^-17.5 a + 2^-18.5 with a = 0.125 sum |q k| (for queries in
whole numbers of 23 bits too: 64 x 2^-22 of the largest |q| and |k| is below 2^-18 of 64 x 0.25 x 0.5); here q <= 1.25,
k <= 1.51, a <= 15.1 (sqrt 2 of it where they are rotated) and e <= 1.2e-4. Numerator and denominator
and both results: 4 e max |v|.
"""
import numpy as np
import pytest

import test_gpu_kv4 as four
import test_gpu_kv8 as eight

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
INF, NAN = float("inf"), float("nan")


def outputs(bits, rows, first, q, t, k, v, rope, lists):
    n = len(k)
    c = eight.Cache(1, 1, (n + 15) // 16) if bits == 8 else four.Cache(1, 1, (n + 15) // 16, 0)
    out = torch.full(q.shape, 7.0, device="cuda:0")
    if bits == 8:
        c.append([n], [0], k, v, "f32")
        r, keep = c.rows([0, rows], [first], rows)
        eight.attend(c, r, q, t, out, "f32", rope=rope, blocks=lists)
    else:
        r, keep = c.rows([0, n], [0], n)
        four.append(c, r, k, v, "f32")
        r, keep = c.rows([0, rows], [first], rows)
        four.attend(c, r, q, t, out, "f32", 0.125, None if rope is None else eight.dev(rope))
    return out


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("bits,listed", [(8, False), (8, True), (4, False)])
@pytest.mark.parametrize("rows,first", [(1, 60), (3, -1), (20, 40), (40, -3), (300, 100)])
def test_queries_that_are_not_finite(t, rope, bits, listed, rows, first):
    """Keys of one sign, so that every product of an infinity is one infinity: scores that are all -Inf are
    no scores of a row that sees nothing."""
    n = max(first + rows, 16)
    k, v = torch.rand(n, 1, 64, device="cuda:0") + 0.5, torch.randn(n, 1, 64, device="cuda:0")
    if first + rows <= 40:
        k[:], v[:] = k[:1], v[:1]
    q = torch.rand(rows, 4, 64, device="cuda:0") + 0.25
    tab = eight.rope_table(n) if rope else None
    lists = eight.dev(np.tile(np.arange((n + 15) // 16, dtype=np.int32), (rows, 1, 1))) if listed else None
    plain = outputs(bits, rows, first, q.to(eight.TYPES[t][1]), t, k, v, tab, lists)
    assert torch.isfinite(plain).all()
    bad = torch.zeros(rows, 4, dtype=torch.bool)
    # (A position and its pair: a rotation turns two infinities to one and a NaN, or two.)
    for i, (row, head, dims, x) in enumerate([(0, 1, [5], -INF), (rows // 2, 2, [63], INF), (rows - 1, 0, [7, 39], -INF),
                                              (rows - 1, 3, [0], NAN), (rows // 3, 0, [33, 2], -INF)]):
        q[row, head, dims] = x
        bad[row, head] = True
    out = outputs(bits, rows, first, q.to(eight.TYPES[t][1]), t, k, v, tab, lists)
    seen = torch.arange(rows) + first >= 0
    want = bad & seen[:, None]
    assert torch.equal(torch.isnan(out).any(-1).cpu(), want) and torch.equal(torch.isnan(out).all(-1).cpu(), want)
    assert ((out - plain)[~want].abs() <= 4 * 1.2e-4 * v.abs().max()).all()
    assert (out[~seen] == 0).all()
