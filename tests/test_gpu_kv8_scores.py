"""Scores of attention over the quantized caches that are large and alike, against fp64
attention over the values that the pages hold.
"""
import numpy as np
import pytest

from paper_2606_12154_amd import hh
from test_gpu_kv8 import TYPES, Cache, attend, dev
import test_gpu_kv4 as four

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def lists_of(rows, pages):
    return dev(np.tile(np.arange(pages, dtype=np.int32), (rows, 1, 1)))


def averages(n, rows, order, seed):
    """Which of n keys score low, values, and what rows at the end get: the mean of the others' values
    that they see.  And the tolerance: weights of one score are the same number, but for two fp16
    terms, 2^-22 of it, and for what brings them to one base: exponentials, 2^-20 each of their
    argument's rounding, a wave's, a split's and the result's.  Sums: n / 32 + 16 roundings of 2^-24 in
    numerator and denominator.  (The low ones' weights are below 2^-20 of the others'.)"""
    rng = np.random.default_rng(seed)
    low = {"alike": np.zeros(n, bool), "low first": np.arange(n) < n - rows - 9, "low last": np.arange(n) >= 37,
           "mixed": rng.random(n) < 0.5}[order]
    low[0] = order == "low first"
    return low, rng.standard_normal((n, 1, 64)).astype(np.float32)


def compare(out, values, low, rows):
    n = len(low)
    want = np.stack([values[np.flatnonzero(~low[:n - rows + i + 1]), 0].mean(0) for i in range(rows)])[:, None]
    tol = np.abs(values).max() * (2 * 2.0 ** -22 + 3 * 2.0 ** -19 + 2 * (n / 32 + 16) * 2.0 ** -24)
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err.max(), tol)


HEADS = torch.tensor([1.0, 0.75, 1.25, 0.5])[:, None]  # of the size
# Rows of a call (of 4 heads: few columns, one tile, several), how many keys there are, a list of them all.
CALLS = [(1, 100, False), (1, 9000, False), (20, 100, False), (64, 700, False), (300, 900, False), (1, 100, True), (30, 700, True)]
ORDERS = ["alike", "low first", "low last", "mixed"]
SIZES = [10.0, 100.0, 1000.0, 10000.0]  # scores up to 2^31 as a power of two


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,n,listed", CALLS)
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("size", SIZES)
def test_equal_scores_have_equal_weights(t, rows, n, listed, order, size):
    """Keys of one score, with others far below it, are averaged, whatever the score's size and wherever
    a wave meets them."""
    low, v = averages(n, rows, order, rows + n)
    k = np.full((n, 1, 64), size, np.float32)
    k[low] = -size
    c = Cache(1, 1, (n + 15) // 16)
    c.append([n], [0], dev(k), dev(v), "f32")
    kk, vv = c.ref.values(0, n)
    assert len(np.unique(np.abs(kk))) == 1
    q = (HEADS * size).repeat(rows, 1, 64).cuda().to(TYPES[t][1])
    r, keep = c.rows([0, rows], [n - rows], rows)
    out = torch.empty(rows, 4, 64, device="cuda:0")
    attend(c, r, q, t, out, "f32", blocks=lists_of(rows, (n + 15) // 16) if listed else None)
    compare(out, vv, low, rows)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,n", [c[:2] for c in CALLS if not c[2]])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("size", SIZES)
def test_equal_scores_of_a_4_bit_cache(t, rows, n, order, size):
    low, v = averages(n, rows, order, rows + n)
    k = np.full((n, 1, 64), size, np.float32)
    k[low] = -size
    c = four.Cache(1, 1, (n + 15) // 16, 0)
    r, keep = c.rows([0, n], [0], n)
    four.append(c, r, dev(k), dev(v), "f32")
    back = [torch.empty(n, 1, 64, device="cuda:0") for _ in "kv"]
    hh.hh_kv4_read(c.desc, r, back[0].data_ptr(), back[1].data_ptr(), hh.HH_F32, 64, 64, torch.cuda.current_stream().cuda_stream)
    assert len(back[0].abs().unique()) == 1
    q = (HEADS * size).repeat(rows, 1, 64).cuda().to(TYPES[t][1])
    r, keep = c.rows([0, rows], [n - rows], rows)
    out = torch.empty(rows, 4, 64, device="cuda:0")
    four.attend(c, r, q, t, out, "f32", 0.125)
    compare(out, back[1].double().cpu().numpy(), low, rows)


@pytest.mark.parametrize("t,top", [("f32", 2.0 ** 127), ("bf16", 2.0 ** 127), ("f16", 2.0 ** 15)])
@pytest.mark.parametrize("rows", [1, 3, 20, 200])
def test_scores_past_fp32_of_a_4_bit_cache(t, top, rows):
    """scale * q . k above 2^128: the largest score takes all, and keys that a query does not see (a product of 0)
    count alike. Weights as in test_gpu_kv8.py: two fp16 terms, 2^-22 each and in their sum, and sums of 2^-24."""
    scale, n = 2.0 ** 100, 205
    rng = np.random.default_rng(2)
    for seen in (True, False):
        k = np.zeros((n, 1, 64), np.float32)
        k[:, 0, 0 if seen else 1] = np.repeat(np.arange(n // 5), 5)[:n] % 41 + 1.0
        k[::7, 0, 0 if seen else 1] *= -1
        k[100, 0, 0 if seen else 1] = 50.0
        v = rng.standard_normal((n, 1, 64)).astype(np.float32)
        c = four.Cache(1, 1, (n + 15) // 16, 0)
        r, keep = c.rows([0, n], [0], n)
        four.append(c, r, dev(k), dev(v), "f32")
        back = [torch.empty(n, 1, 64, device="cuda:0") for _ in "kv"]
        hh.hh_kv4_read(c.desc, r, back[0].data_ptr(), back[1].data_ptr(), hh.HH_F32, 64, 64, torch.cuda.current_stream().cuda_stream)
        q = torch.zeros(rows, 4, 64, device="cuda:0")
        q[:, :, 0] = top
        r, keep = c.rows([0, rows], [n - rows], rows)
        out = torch.empty(rows, 4, 64, device="cuda:0")
        four.attend(c, r, q.to(TYPES[t][1]), t, out, "f32", scale)
        kk, vv = (a.double().cpu().numpy()[:, 0] for a in back)
        for i in range(rows):
            m = n - rows + i + 1
            best = np.flatnonzero(kk[:m, 0] == kk[:m, 0].max())
            want = vv[best].mean(0)
            err = np.abs(out[i].double().cpu().numpy() - want)
            assert (err <= np.abs(vv).max() * (2 * 2.0 ** -22 + (m / 32 + 16) * 2.0 ** -23 + 3 * 2.0 ** -19)).all(), (seen, i, err.max())


@pytest.mark.parametrize("t,rope", [("f32", False), ("f16", False), ("bf16", False), ("f32", True)])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows", [1, 4, 40, 300])
def test_large_scores_that_differ_by_little(t, rope, bits, rows):
    """Scores of 2^18 to 2^30 as a power of two, which rise by 1/4 to 100 from page to page (a dimension of small
    queries whose keys rise): beside the rounding of such scores any of the higher ones may take all, but weights
    stay finite, and results a mean of the values.  The bound: a mean's, and of its two fp16 terms and sums."""
    torch.manual_seed(0)
    n = 700
    sizes = torch.exp2(torch.linspace(8, 14.5, 4 * rows)).reshape(rows, 4, 1)  # |q| = |k| times a constant
    steps = torch.exp2(torch.rand(rows, 4) * 9 - 3)
    k, v = torch.full((n, 1, 64), 512.0), torch.randn(n, 1, 64).abs() + 0.5
    k[:, 0, 31] = (torch.arange(n) // 16 % 5 * 128).float()
    k[:, 0, 63] = 0.0
    # (A rise of 128 in the 31st dimension: steps as a power of two; the pair's other dimension is 0.)
    q = (sizes.square() / 512).expand(rows, 4, 64).clone()
    q[..., 31], q[..., 63] = steps / (128 * 0.125 * 1.4427), 0.0
    if t == "f16":
        q = q.clamp(max=60000.0)
    tab = torch.tensor([1.0, 0.0]).expand(n, 32, 2).contiguous().cuda() if rope else None
    q, k, v = (x.cuda().contiguous() for x in (q.to(TYPES[t][1]), k, v))
    out = torch.empty(rows, 4, 64, device="cuda:0")
    if bits == 8:
        c = Cache(1, 1, (n + 15) // 16)
        c.append([n], [0], k, v, "f32", ref=False)
        r, keep = c.rows([0, rows], [n - rows], rows)
        attend(c, r, q, t, out, "f32", rope=None if tab is None else tab.cpu().numpy())
    else:
        c = four.Cache(1, 1, (n + 15) // 16, 0)
        r, keep = c.rows([0, n], [0], n)
        four.append(c, r, k, v, "f32")
        r, keep = c.rows([0, rows], [n - rows], rows)
        four.attend(c, r, q, t, out, "f32", 0.125, tab)
    most, least = v.max() * (1 + (1 / 14 if bits == 4 else 1 / 250)), v.min() - v.max() / (14 if bits == 4 else 250)
    slack = v.max() * (2.0 ** -21 + (n / 32 + 16) * 2.0 ** -23)
    assert torch.isfinite(out).all()
    assert (out <= most + slack).all() and (out >= least - slack).all()
