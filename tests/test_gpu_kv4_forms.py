"""Attention over the 4-bit paged cache: its error in every pairing of element
types, element by element, against fp64 attention over the values that the pages hold.

Bound of an element, whatever kernel a call takes, with s = sum of w |v| over the attended
keys, a = scale * sum of |q_i k_i| of the row's key where that is largest (|q_i| of a rotated
query: the length of the pair it is rotated in, which no rotation changes), n keys, m = max |v|:
  - scores: queries hold 22 bits (2^-22 of each product); the sums of 64 products take 64 fp32
    roundings (2^-18 of a), a rotation 3 * 2^-24, scaling and base 4 * 2^-24 and one 2^-24
    more for each time the base is raised (24 of them counted): 2^-17.5 a in all;
  - a weight: the exponential's 2^-23 and its argument's rounding, 2^-24 of less than 2^5, and
    22 bits: 2^-18.5;
  - so each weight is off by e = 2^-17.5 a + 2^-18.5, numerator and denominator both: 2 e s;
    sums over the keys, 32 at a time, n / 32 roundings each and 16 for joins: 2 (n / 32 + 16) 2^-24 s;
  - the smallest weights are off by half the lowest step of fp16, 2^-25, where the largest
    is 2^12 or more: 2^-37 of the largest, and so of the sum, n times, in both: 2^-36 n m;
  - then half a step of the output's type.
One fp16 number for a weight or a rotated query is up to 2^-12 of it off, 2^-12 a for the query, and
passes this bound in rows of few keys.
"""
import numpy as np
import pytest

from oracle import kv4
from kv4_cases import CASES
from test_gpu_kv4 import TYPES, Cache, append, attend, dev, rope_table

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def reference(q, k, v, scale, pos, length):
    """fp64 rows [n, heads, 64] at positions pos [n] over k and v [keys, kv heads, 64];
    length: |q| for a. Returns the results and s and a."""
    n, hq, _ = q.shape
    keys, hkv, _ = k.shape
    g = hq // hkv
    out, s, a = torch.empty_like(q), torch.empty_like(q), torch.empty(n, hq, 1, dtype=torch.float64, device=q.device)
    hidden = torch.arange(keys, device=q.device)[None] > pos[:, None]
    for h in range(hq):
        kh, vh = k[:, h // g].contiguous(), v[:, h // g].contiguous()
        x = (q[:, h].contiguous() @ kh.T.contiguous() * scale).masked_fill(hidden, -np.inf)
        w = torch.softmax(x, -1)
        out[:, h], s[:, h] = w @ vh, w @ vh.abs()
        a[:, h, 0] = (length[:, h].contiguous() @ kh.abs().T.contiguous() * scale).masked_fill(hidden, 0).amax(-1)
    return out, s, a


def check(got, q, k, v, scale, pos, ot, rope=None):
    """The docstring's bound for rows `got` (fp64) of queries q (before their rotation)."""
    length = q.abs()
    if rope is not None:
        c, s = rope[pos.long()].double().unbind(-1)
        c, s, x, y = c[:, None], s[:, None], q[..., :32], q[..., 32:]
        length = torch.sqrt(x * x + y * y).repeat(1, 1, 2)
        q = torch.cat([x * c - y * s, y * c + x * s], -1)
    ref, s, a = reference(q, k, v, scale, pos, length)
    n = (pos + 1).double()[:, None, None]
    e = 2.0 ** -17.5 * a + 2.0 ** -18.5
    e = (2 * e + 2 * (n / 32 + 16) * 2.0 ** -24) * s + 2.0 ** -36 * n * v.abs().max()
    tol = e + HALF_STEP[ot] * (ref.abs() + e) + 2.0 ** -25
    assert torch.isfinite(got).all()
    over = ((got - ref).abs() - tol).amax().item()
    worst = ((got - ref).abs() / tol).amax().item()
    assert over <= 0, f"an element is {worst:.3g} times the bound off ({over:.3g} over it)"
    return worst


def run(rows, first, hkv, group, t, ot, rope, seed, max_pages=None, scale=0.125, sample=None):
    """rows[i] rows of sequence i from position first[i] on; sample: rows compared of each."""
    torch.manual_seed(seed)
    lens = [r + f for r, f in zip(rows, first)]
    c = Cache(len(lens), hkv, max_pages or (max(lens) + 15) // 16, seed)
    n, hq = sum(lens), hkv * group
    at = np.concatenate([[0], np.cumsum(lens)])
    x = [torch.randn(n, hkv, 64, device="cuda:0") for _ in "kv"]
    r, keep = c.rows(at, [0] * len(lens), n)
    append(c, r, *x, "f32")
    held = [torch.empty_like(a) for a in x]
    from paper_2606_12154_amd import hh
    hh.hh_kv4_read(c.desc, r, held[0].data_ptr(), held[1].data_ptr(), hh.HH_F32, hkv * 64, hkv * 64,
                   torch.cuda.current_stream().cuda_stream)
    k, v = (a.double() for a in held)
    start = np.concatenate([[0], np.cumsum(rows)])
    q = torch.randn(int(start[-1]), hq, 64, device="cuda:0").to(TYPES[t][1])
    out = torch.full(q.shape, 3.0, dtype=TYPES[ot][1], device="cuda:0")
    tab = dev(rope_table(max(lens))) if rope else None
    r, keep = c.rows(start, first, int(start[-1]))
    attend(c, r, q, t, out, ot, scale, tab)
    worst = 0.0
    for i in range(len(rows)):
        which = torch.arange(rows[i], device="cuda:0")
        if sample and rows[i] > sample:  # the first, the last, and others between them
            some = torch.randperm(rows[i] - 1, device="cuda:0")[:sample - sample // 2 - 1]
            which = torch.cat([torch.arange(sample // 2, device="cuda:0"), some, which[-1:]])
        at_row = which + int(start[i])
        worst = max(worst, check(out[at_row].double(), q[at_row].double(), k[at[i]:at[i + 1]], v[at[i]:at[i + 1]], scale,
                                 which + first[i], ot, tab))
    return worst


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("ot", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_single_tokens_of_few_keys(t, ot, rope):
    """Rows of 1 to 6 keys, where one rounded weight or query shows."""
    n = 600
    run([1] * n, [i % 6 for i in range(n)], 2, 4, t, ot, rope, seed=1)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("ot", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_prompts_of_many_rows(t, ot, rope):
    """The first rows of prompts have few keys, and their tiles many columns."""
    run([1400, 9, 700], [0, 2, 0], 4, 4, t, ot, rope, seed=2, sample=64)
    run([40] * 24, [i % 3 for i in range(24)], 8, 4, t, ot, rope, seed=3)


@pytest.mark.parametrize("rows,seqs", [(1, 1024), (20, 512)])
@pytest.mark.parametrize("ot", ["f32", "bf16"])
def test_many_small_weights(rows, seqs, ot):
    """20,000 flat keys behind steep ones, one in each wave's first pages (so many sequences of one
    table row that no range is split). Steep keys have the value 0, the others 7, and weights
    2^-x of the steep ones': the result is 7 n 2^-x over the steep keys' number and that sum. Beside
    2 (n / 32 + 16 + 64) 2^-24 of it (sums as in check(), and a score of 7 b log2 e < 2^6 whose
    two roundings the exponent takes as they are), 2^-37 of the largest weight may be lost n times."""
    n, steep = 20000, torch.arange(8) * 32
    k, v = torch.zeros(n, 1, 64, device="cuda:0"), torch.full((n, 1, 64), 7.0, device="cuda:0")
    k[steep, 0, 0], v[steep] = 7.0, 0.0
    c = Cache(1, 1, n // 16)
    r, keep = c.rows([0, n], [0], n)
    append(c, r, k, v, "f32")
    x = torch.arange(30, 42, dtype=torch.float64)
    b = (x * np.log(2.0) / 7).float()
    q = torch.zeros(seqs * rows, 12, 64, device="cuda:0")
    q[..., 0] = dev(b)
    out = torch.full(q.shape, 9.0, dtype=TYPES[ot][1], device="cuda:0")
    first = n - rows
    r, keep = c.rows(np.arange(seqs + 1) * rows, [first] * seqs, seqs * rows, table_row=np.zeros(seqs))
    attend(c, r, q, "f32", out, ot, 1.0)
    w = torch.exp(-7 * b.double())
    for i in {0, rows - 1}:
        flat = first + i + 1 - len(steep)
        ref = 7 * flat * w / (len(steep) + flat * w)
        tol = 2 * (n / 32 + 80) * 2.0 ** -24 * ref + 2.0 ** -37 * 7 * flat / len(steep)
        tol += HALF_STEP[ot] * (ref + tol)
        got = out.view(seqs, rows, 12, 64)[:, i].double().cpu()
        err = (got - ref[:, None]).abs() / tol[:, None]
        assert err.max() <= 1, [f"2^-{int(a)}: {e:.3g}" for a, e in zip(x, err.amax((0, 2)))]


@pytest.mark.parametrize("t,ot,rope", [("f16", "f16", False), ("bf16", "bf16", False), ("f32", "f32", False),
                                       ("f32", "bf16", False), ("bf16", "bf16", True), ("f32", "f16", True)])
@pytest.mark.parametrize("case", list(CASES))
def test_every_kernel(case, t, ot, rope):
    """Queries of one and of two terms through every kernel and way of cutting a call up."""
    rows, first, hkv, group, pages = CASES[case]
    run(rows, first, hkv, group, t, ot, rope, seed=7, max_pages=pages, sample=40)
