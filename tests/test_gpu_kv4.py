"""The 4-bit paged cache's operators on the GPU against the fp64 oracle.

* Appended bytes and values read back are exact (integer and fp16 work; keys are
  rotated in 64 bits and rounded once), and only the given slots are written.
* Attention is compared with fp64 attention over the values that the pages hold.
  Its bound, for every element (a = max over the attended keys of
  scale * sum |q_i k_i|, m = max |v|):
    - scores: queries as fp16 terms, 2^-22 of each product, and 64 fp32 sums,
      2^-18 of sum |q k|; a rotation in fp32, 3 * 2^-24 more; the power's argument
      and the exponential, 2^-20 and 2^-21 of a weight (|argument| < 2^7):
      e = 2^-17.5 a + 2^-19;
    - weights relative to their sum: 2 e, with 16-bit outputs 2 * 2^-12 more, and
      with fp32 ones 2 * 2^-22; sums of n weights and products in fp32: pairs of
      pages at 2^-24 each, n / 32 of them at most, here below 2^-17;
    - so |out - ref| <= m (2 e + 2 w + 2^-17) + half a step of the output's type.
* Pools start as 0xff bytes, so that every slot that no row may read holds NaN.
"""
import numpy as np
import pytest

from oracle import kv4
from paper_2606_12154_amd import hh

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f32": (hh.HH_F32, torch.float32), "f16": (hh.HH_F16, torch.float16), "bf16": (hh.HH_BF16, torch.bfloat16)}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
WEIGHT = {"f32": 2.0 ** -22, "f16": 2.0 ** -12, "bf16": 2.0 ** -12}


def dev(a, dtype=None):
    return torch.as_tensor(a, dtype=dtype, device="cuda:0")


def ints(a):
    return dev(np.asarray(a, dtype=np.int32))


def rope_table(n):
    ang = np.arange(n)[:, None] * 1e4 ** (-np.arange(32) / 32.0)
    return np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)


class Cache:
    """A pool of 0xff bytes with a shuffled page for every slot of the table."""

    def __init__(self, seqs, hkv, max_pages, seed=0, spare=3):
        self.hkv, self.max_pages = hkv, max_pages
        n = seqs * max_pages
        self.n_pages = n + spare
        self.table = np.random.default_rng(seed).permutation(self.n_pages)[:n].reshape(seqs, max_pages).astype(np.int32)
        self.pool = torch.full((self.n_pages, hkv, kv4.BLOCK), 255, dtype=torch.uint8, device="cuda:0")
        self.d_table = ints(self.table)
        self.desc = hh.hh_kv4_pool(self.pool.data_ptr(), self.d_table.data_ptr(), self.n_pages, hkv, max_pages, seqs)

    def rows(self, start, first, n_rows, table_row=None):
        keep = [None if a is None else ints(a) for a in (start, first, table_row)]
        longest = 1 if start is None else max(1, int(np.diff(start).max()))
        r = hh.hh_kv4_rows(*[None if t is None else t.data_ptr() for t in keep], len(first), n_rows, longest)
        return r, keep


def stream():
    return torch.cuda.current_stream().cuda_stream


def append(c, r, k, v, t, rope=None):
    hh.hh_kv4_append(c.desc, r, k.data_ptr(), v.data_ptr(), TYPES[t][0], k.stride(0), v.stride(0),
                     None if rope is None else rope.data_ptr(), 0 if rope is None else rope.shape[0], stream())


def attend(c, r, q, t, out, ot, scale=0.125, rope=None, ws=None):
    hq = q.shape[1]
    need = hh.hh_kv4_attention_workspace(c.desc, r, hq)
    if ws is None:
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda:0")
    hh.hh_kv4_attention(c.desc, r, q.data_ptr(), TYPES[t][0], q.stride(0), hq, scale,
                        None if rope is None else rope.data_ptr(), 0 if rope is None else rope.shape[0],
                        out.data_ptr(), TYPES[ot][0], out.stride(0), ws.data_ptr() if need else None, ws.numel(), stream())
    return ws


# ------------------------------------------------------------------ append and read

def special(x, rng):
    """Rows on the format's borders among ordinary ones [n, heads, 64]."""
    n = x.shape[0]
    for i, f in enumerate([lambda a: a * 0, lambda a: a * 1e-7, lambda a: a * 2.0 ** -15, lambda a: a * 3e4,
                           lambda a: np.where(np.arange(64) % 2, 7.0, 2.5 * np.sign(a)), lambda a: a * 1e-30]):
        if n > 2 * i:
            x[2 * i, 0] = f(x[2 * i, 0])
    return x


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("lens,first", [([1], [0]), ([1, 1, 1], [5, 16, 31]), ([40, 3], [0, 14]), ([17, 1, 33], [15, 47, 1])])
def test_append_bytes_and_read(t, rope, lens, first):
    rng = np.random.default_rng(len(lens) + first[0])
    hkv, n = 3, sum(lens)
    c = Cache(len(lens), hkv, 4)
    start = np.concatenate([[0], np.cumsum(lens)])
    wide = torch.zeros((n, 2 * hkv + 1, 64), dtype=TYPES[t][1], device="cuda:0")
    wide[:, :hkv] = dev(special(rng.standard_normal((n, hkv, 64)), rng), torch.float32).to(TYPES[t][1])
    wide[:, hkv:2 * hkv] = dev(special(rng.standard_normal((n, hkv, 64)), rng), torch.float32).to(TYPES[t][1])
    k, v = wide[:, :hkv], wide[:, hkv:2 * hkv]
    tab = rope_table(64)
    d_tab = dev(tab)
    r, keep = c.rows(start, first, n)
    append(c, r, k, v, t, d_tab if rope else None)
    kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
    pos = np.concatenate([f + np.arange(m) for f, m in zip(first, lens)])
    seq = np.repeat(np.arange(len(lens)), lens)
    if rope:
        kf = kv4.rotate(kf, tab, pos).astype(np.float32)
    want = np.full((c.n_pages, hkv, kv4.BLOCK), 255, np.uint8)
    for i in range(n):
        for h in range(hkv):
            kv4.put(want[c.table[seq[i], pos[i] // 16], h], pos[i] % 16, kf[i, h], vf[i, h])
    assert np.array_equal(c.pool.cpu().numpy(), want)
    back = [torch.full((n, hkv, 64), 9.0, dtype=TYPES[t][1], device="cuda:0") for _ in "kv"]
    hh.hh_kv4_read(c.desc, r, back[0].data_ptr(), back[1].data_ptr(), TYPES[t][0], hkv * 64, hkv * 64, stream())
    for got, x in zip(back, (kf, vf)):
        ref = torch.from_numpy(kv4.values(x)).to(TYPES[t][1])
        # (fp16 holds one special row as infinities: NaN, by definition.)
        assert np.array_equal(got.double().cpu().numpy(), ref.double().numpy(), equal_nan=True)


@pytest.mark.parametrize("hkv", [3, 5, 8])
def test_many_rows_of_several_heads_a_workgroup(hkv):
    lens, first = [4000, 1, 1700, 33], [3, 40, 0, 15]
    n = sum(lens)
    c = Cache(4, hkv, 256)
    k, v = (torch.randn(n, hkv, 64, device="cuda:0") for _ in "kv")
    r, keep = c.rows(np.concatenate([[0], np.cumsum(lens)]), first, n)
    append(c, r, k, v, "f32")
    back = [torch.full_like(k, 9.0) for _ in "kv"]
    hh.hh_kv4_read(c.desc, r, back[0].data_ptr(), back[1].data_ptr(), hh.HH_F32, hkv * 64, hkv * 64, stream())
    for got, x in zip(back, (k, v)):
        assert np.array_equal(got.double().cpu().numpy(), kv4.values(x.cpu().numpy()))
    held = (c.pool != 255).any(-1).all(-1).sum().item()
    assert held == sum((f + m - 1) // 16 - f // 16 + 1 for f, m in zip(first, lens))


def test_rows_that_are_not_finite_read_as_nan():
    c = Cache(1, 2, 2)
    k, v = (torch.randn(20, 2, 64, device="cuda:0") for _ in "kv")
    k[3, 1, 40], v[7, 0, 1], v[8, 1, 63] = float("nan"), float("inf"), -float("inf")
    r, keep = c.rows([0, 20], [0], 20)
    append(c, r, k, v, "f32")
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    hh.hh_kv4_read(c.desc, r, kb.data_ptr(), vb.data_ptr(), hh.HH_F32, 128, 128, stream())
    for got, bad in ((kb, [(3, 1)]), (vb, [(7, 0), (8, 1)])):
        nan = torch.isnan(got.cpu())
        want = torch.zeros_like(nan)
        for i, h in bad:
            want[i, h] = True
        assert torch.equal(nan, want)


def test_padding_and_places_past_the_table():
    """Rows at negative positions and past the table or the rotation's are
    skipped by append and read as 0; a table row out of range has no page."""
    c = Cache(2, 1, 2)
    n = 8
    k, v = (torch.randn(n, 1, 64, device="cuda:0") for _ in "kv")
    # Sequences: 3 rows at -2, -1, 0; 3 rows at 30 .. 32 (the table ends at 32);
    # one row of table row 7, one of table row -1.
    r, keep = c.rows([0, 3, 6, 7, 8], [-2, 30, 0, 0], n, table_row=[0, 1, 7, -1])
    append(c, r, k, v, "f32")
    kb, vb = (torch.full((n, 1, 64), 5.0, device="cuda:0") for _ in "kv")
    hh.hh_kv4_read(c.desc, r, kb.data_ptr(), vb.data_ptr(), hh.HH_F32, 64, 64, stream())
    for got, x in ((kb, k), (vb, v)):
        want = kv4.values(x.cpu().numpy())
        want[[0, 1, 5, 6, 7]] = 0
        assert np.array_equal(got.cpu().numpy(), want.astype(np.float32))
    held = (c.pool != 255).any(-1).nonzero().cpu().numpy()[:, 0].tolist()
    assert sorted(held) == sorted([c.table[0, 0], c.table[1, 1]])
    # A rotation table that ends before the rows: those are skipped.
    c2 = Cache(1, 1, 2)
    tab = dev(rope_table(4))
    r2, keep2 = c2.rows([0, 8], [0], 8)
    append(c2, r2, k, v, "f32", tab)
    hh.hh_kv4_read(c2.desc, r2, kb.data_ptr(), vb.data_ptr(), hh.HH_F32, 64, 64, stream())
    assert torch.isfinite(kb[:4]).all() and torch.isnan(kb[4:]).all()


# ------------------------------------------------------------------ attention

def filled(lens, hkv, seed, max_pages=None):
    """A cache that holds lens[i] positions of sequence i, and the fp64 values."""
    rng = np.random.default_rng(seed)
    c = Cache(len(lens), hkv, max_pages or max(1, (max(lens) + 15) // 16), seed)
    n = sum(lens)
    x = [rng.standard_normal((n, hkv, 64)).astype(np.float32) for _ in "kv"]
    if n:
        start = np.concatenate([[0], np.cumsum(lens)])
        r, keep = c.rows(start, [0] * len(lens), n)
        append(c, r, dev(x[0]), dev(x[1]), "f32")
    at = np.concatenate([[0], np.cumsum(lens)])
    return c, [[kv4.values(a[at[i]:at[i + 1]]) for a in x] for i in range(len(lens))]


def check(got, q, k, v, scale, first, ot, rope_err=0.0):
    """got [n, heads, 64] fp64 against the bound of the module's docstring."""
    ref = kv4.attend(q, k, v, scale, first)
    n, hq = q.shape[:2]
    group = hq // k.shape[1]
    a = 0.0
    for h in range(hq):
        a = max(a, float((np.abs(q[:, h]) @ np.abs(k[:, h // group]).T).max(initial=0.0)) * scale)
    m = float(np.abs(v).max(initial=0.0))
    e = 2.0 ** -17.5 * a + 2.0 ** -19
    tol = m * (2 * e + 2 * WEIGHT[ot] + 2.0 ** -17) + HALF_STEP[ot] * np.abs(ref) + 2.0 ** -25
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= tol).all(), f"{err.max():.3g} off, {np.max(err - tol):.3g} over the bound"


def run_case(lens, rows, hkv, group, t, ot, rope, seed, scale=0.125):
    """rows[i] query rows that end the i-th sequence of lens[i] positions."""
    c, kv = filled(lens, hkv, seed)
    rng = np.random.default_rng(seed + 1)
    n, hq = sum(rows), hkv * group
    wide = torch.zeros((n + 1, hq + 1, 64), dtype=TYPES[t][1], device="cuda:0")
    wide[:n, :hq] = dev(rng.standard_normal((n, hq, 64)), torch.float32).to(TYPES[t][1])
    q = wide[:, :hq]
    out = torch.full((n + 1, hq + 2, 64), 3.0, dtype=TYPES[ot][1], device="cuda:0")
    start = np.concatenate([[0], np.cumsum(rows)])
    first = [a - b for a, b in zip(lens, rows)]
    r, keep = c.rows(start, first, n + 1)
    tab = rope_table(max(lens) + 1)
    attend(c, r, q, t, out, ot, scale, dev(tab) if rope else None)
    got = out.double().cpu().numpy()
    assert (got[n] == 3.0).all() and (got[:, hq:] == 3.0).all(), "rows in no sequence and other columns stay"
    qf = q.double().cpu().numpy()
    for i in range(len(lens)):
        qi = qf[start[i]:start[i + 1]]
        if rope:
            qi = kv4.rotate(qi, tab, np.maximum(first[i] + np.arange(rows[i]), 0))
        check(got[start[i]:start[i + 1], :hq], qi, kv[i][0], kv[i][1], scale, first[i], ot)


@pytest.mark.parametrize("t,ot", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("lens", [[1], [2, 15, 16, 17], [31, 32, 33, 300], [700, 64]])
def test_single_tokens(t, ot, rope, lens):
    run_case(lens, [1] * len(lens), 2, 4, t, ot, rope, seed=sum(lens))


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16, 17, 40])
def test_head_groups(group):
    run_case([37, 5], [1, 1], 3, group, "f16", "f16", False, seed=group)
    run_case([37, 50], [9, 1], 1, group, "f32", "f32", True, seed=group)


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("lens,rows", [([5, 40], [5, 1]), ([40, 3, 90], [7, 3, 13]), ([100], [100]), ([230, 77], [150, 77])])
def test_several_rows(t, lens, rows):
    run_case(lens, rows, 2, 4, t, t, len(lens) == 2, seed=sum(rows))


def test_wide_tiles():
    """Enough rows that a wave keeps its columns to itself (no key splits)."""
    run_case([300] * 13, [260] * 12 + [31], 8, 4, "f16", "f16", False, seed=9)


def test_long_tokens_split_over_keys():
    run_case([5000, 3, 2049], [1, 1, 1], 1, 2, "f16", "f16", False, seed=5)
    run_case([4111], [3], 1, 8, "f32", "f32", True, seed=6)


def test_more_sequences_than_a_launch_takes():
    """1,100 sequences of up to 2^20 rows by the description (most have none):
    2^32 threads and more, which two launches of each call share."""
    n_seqs, most = 1100, 1 << 20
    lens = np.zeros(n_seqs, int)
    lens[[0, 7, 1022, 1023, 1024, 1099]] = [3, 1, 4, 2, 1, 5]
    start = np.concatenate([[0], np.cumsum(lens)])
    n = int(start[-1])
    c = Cache(n_seqs, 1, 2)
    rng = np.random.default_rng(11)
    k, v = (rng.standard_normal((n, 1, 64)).astype(np.float32) for _ in "kv")
    keep = [ints(start), ints(np.zeros(n_seqs))]
    r = hh.hh_kv4_rows(keep[0].data_ptr(), keep[1].data_ptr(), None, n_seqs, n, most)
    append(c, r, dev(k), dev(v), "f32")
    back = [torch.full((n, 1, 64), 9.0, device="cuda:0") for _ in "kv"]
    hh.hh_kv4_read(c.desc, r, back[0].data_ptr(), back[1].data_ptr(), hh.HH_F32, 64, 64, stream())
    for got, x in zip(back, (k, v)):
        assert np.array_equal(got.double().cpu().numpy(), kv4.values(x))
    q = torch.randn(n, 1, 64, device="cuda:0")
    out = torch.full_like(q, 9.0)
    attend(c, r, q, "f32", out, "f32")
    got, qf = out.double().cpu().numpy(), q.double().cpu().numpy()
    for i in np.flatnonzero(lens):
        rows = slice(start[i], start[i + 1])
        check(got[rows], qf[rows], kv4.values(k[rows]), kv4.values(v[rows]), 0.125, 0, "f32")


@pytest.mark.parametrize("seqs,most,hkv,group,t,ot", [(1, 700, 8, 4, "f16", "f16"), (24, 640, 8, 2, "bf16", "bf16"), (40, 1300, 2, 7, "f32", "f32"), (3, 1500, 4, 4, "f32", "f16")])
def test_tokens_of_ragged_lengths(seqs, most, hkv, group, t, ot):
    """Lengths from one position to the longest, with wide workgroups and with splits that only the long ones reach."""
    lens = [most] + [1 + (most - 1) * i // seqs for i in range(seqs - 1)]
    run_case(lens, [1] * seqs, hkv, group, t, ot, seqs == 24, seed=seqs)


@pytest.mark.parametrize("rows,seqs", [(1, 1024), (20, 512)])
def test_long_ranges_that_are_not_split(rows, seqs):
    """So many sequences (of one table row) that each workgroup takes its whole
    range: up to 160 steps a wave, whose fp32 sums add 160 * 2^-24 of the weights and of
    the products, < 2^-15.6, to check()'s bound (which counts them as 2^-17)."""
    n = 20000
    c, kv = filled([n], 1, 21)
    rng = np.random.default_rng(rows)
    first = rng.integers(8000, n - rows, seqs)
    first[:3] = [n - rows, 8192, 8191]
    q = dev(rng.standard_normal((seqs * rows, 2, 64)), torch.float32)
    out = torch.full_like(q, 9.0)
    r, keep = c.rows(np.arange(seqs + 1) * rows, first, seqs * rows, table_row=np.zeros(seqs))
    assert hh.hh_kv4_attention_workspace(c.desc, r, 2) == 0
    attend(c, r, q, "f32", out, "f32")
    k, v = kv[0]
    more = float(np.abs(v).max()) * 2.0 ** -15.6
    for s in range(16):
        at = slice(s * rows, s * rows + rows)
        qs, got = q[at].double().cpu().numpy(), out[at].double().cpu().numpy()
        ref = kv4.attend(qs, k, v, 0.125, int(first[s]))
        check(got - np.clip(got - ref, -more, more), qs, k, v, 0.125, int(first[s]), "f32")


def test_scales_of_scores():
    """Steep and flat softmaxes, and queries far from 1."""
    run_case([200], [2], 1, 4, "f32", "f32", False, seed=7, scale=2.0)
    run_case([200], [2], 1, 4, "f32", "f32", False, seed=8, scale=1e-4)
    c, kv = filled([90], 1, 3)
    for f in (1e-20, 1e18, 0.0):
        q = torch.randn(1, 2, 64, device="cuda:0") * f
        out = torch.empty_like(q)
        r, keep = c.rows([0, 1], [89], 1)
        scale = float(min(max(0.125 / f, 1e-30), 1e30)) if f else 1.0
        attend(c, r, q, "f32", out, "f32", scale)
        check(out.double().cpu().numpy(), q.double().cpu().numpy(), *kv[0], np.float32(scale).astype(float), 89, "f32")


def test_tiny_and_large_values():
    """Values near the ends of the format's range keep their relative precision."""
    for f in (1e-6, 1e-4, 2000.0):
        c = Cache(1, 1, 3)
        rng = np.random.default_rng(4)
        k = rng.standard_normal((48, 1, 64)).astype(np.float32)
        v = (f * rng.standard_normal((48, 1, 64))).astype(np.float32)
        r, keep = c.rows([0, 48], [0], 48)
        append(c, r, dev(k), dev(v), "f32")
        q = torch.randn(1, 4, 64, device="cuda:0")
        out = torch.empty_like(q)
        r, keep = c.rows([0, 1], [47], 1)
        attend(c, r, q, "f32", out, "f32")
        ref = kv4.attend(q.double().cpu().numpy(), kv4.values(k), kv4.values(v), 0.125, 47)
        m = float(np.abs(kv4.values(v)).max())
        assert np.abs(out.double().cpu().numpy() - ref).max() <= m * 2.0 ** -12


def test_rows_that_see_nothing_are_zero():
    c, kv = filled([20], 2, 1)
    q = torch.randn(7, 4, 64, device="cuda:0", dtype=torch.float16)
    out = torch.full_like(q, 3.0)
    # 4 rows at -2 .. 1, 2 padding rows, and a sequence without rows.
    r, keep = c.rows([0, 4, 4, 5, 6], [-2, 3, -1, -50], 7, table_row=[0, 0, 0, 0])
    attend(c, r, q, "f16", out, "f16")
    got = out.double().cpu().numpy()
    assert (got[[0, 1, 4, 5]] == 0).all() and (got[6] == 3).all()
    check(got[2:4], q[2:4].double().cpu().numpy(), *kv[0], 0.125, 0, "f16")
    # A table row out of range: nothing to attend to.
    r, keep = c.rows([0, 1, 2], [3, 3], 7, table_row=[5, -1])
    attend(c, r, q, "f16", out, "f16")
    assert (out[:2] == 0).all()


@pytest.mark.parametrize("rows,group", [(2, 2), (4, 2), (3, 5), (2, 1)])
@pytest.mark.parametrize("n", [5, 16, 17, 30, 33, 50, 64, 65, 300])
@pytest.mark.parametrize("t", ["f16", "f32"])
def test_nan_in_the_last_position_of_few_rows(rows, group, n, t):
    """Only the last row attends to a key (head 0) or a value (head 1) that is
    not finite: the others, whose keys share operands with it, are exact."""
    c = Cache(1, 2, (n + 15) // 16)
    rng = np.random.default_rng(n)
    k, v = (rng.standard_normal((n, 2, 64)).astype(np.float32) for _ in "kv")
    k[n - 1, 0, 40], v[n - 1, 1, 3] = np.inf, np.nan
    r, keep = c.rows([0, n], [0], n)
    append(c, r, dev(k), dev(v), "f32")
    q = torch.randn(rows, 2 * group, 64, device="cuda:0").to(TYPES[t][1])
    out = torch.empty_like(q)
    r, keep = c.rows([0, rows], [n - rows], rows)
    attend(c, r, q, t, out, t)
    got, qf = out.double().cpu().numpy(), q.double().cpu().numpy()
    assert np.isnan(got[-1]).all()
    kz, vz = kv4.values(np.nan_to_num(k, posinf=0)), kv4.values(np.nan_to_num(v))
    check(got[:-1], qf[:-1], kz, vz, 0.125, n - rows, t)


@pytest.mark.parametrize("rows", [30, 200])
@pytest.mark.parametrize("t", ["f16", "f32"])
def test_nan_reaches_only_rows_that_attend_to_it(rows, t):
    """A key and a value row that are not finite: rows before them are exact."""
    n = 70 + rows
    c = Cache(1, 2, (n + 15) // 16)
    rng = np.random.default_rng(rows)
    k, v = (rng.standard_normal((n, 2, 64)).astype(np.float32) for _ in "kv")
    bad_k, bad_v = n - rows // 2, n - rows // 3
    k[bad_k, 0, 3], v[bad_v, 1, 60] = np.nan, np.inf
    r, keep = c.rows([0, n], [0], n)
    append(c, r, dev(k), dev(v), "f32")
    q = torch.randn(rows, 4, 64, device="cuda:0").to(TYPES[t][1])
    out = torch.empty_like(q)
    r, keep = c.rows([0, rows], [n - rows], rows)
    attend(c, r, q, t, out, t)
    got, qf = out.double().cpu().numpy(), q.double().cpu().numpy()
    pos = n - rows + np.arange(rows)
    nan = np.isnan(got)
    assert np.array_equal(nan.all(-1), nan.any(-1))
    assert np.array_equal(nan[:, :2, 0], np.repeat((pos >= bad_k)[:, None], 2, 1))
    assert np.array_equal(nan[:, 2:, 0], np.repeat((pos >= bad_v)[:, None], 2, 1))
    kz, vz = kv4.values(np.nan_to_num(k, posinf=0)), kv4.values(np.nan_to_num(v, posinf=0))
    m = bad_k - (n - rows)
    check(got[:m], qf[:m], kz, vz, 0.125, n - rows, t)


def test_page_ids_out_of_range_stay_inside_the_pool():
    """Such an id is refused by append and taken as page 0 by the readers."""
    c, kv = filled([16], 1, 2)
    before = c.pool.clone()
    c.d_table.fill_(1 << 30)
    r, keep = c.rows([0, 1], [3], 1)
    k = torch.randn(1, 1, 64, device="cuda:0")
    append(c, r, k, k, "f32")
    assert torch.equal(c.pool, before)
    q, out = torch.randn(1, 1, 64, device="cuda:0"), torch.empty(1, 1, 64, device="cuda:0")
    attend(c, r, q, "f32", out, "f32")
    torch.cuda.synchronize()


def test_repeats_streams_and_graphs_give_the_same_bits():
    c, kv = filled([900, 33], 2, 11)
    q = torch.randn(2, 8, 64, device="cuda:0", dtype=torch.float16)
    r, keep = c.rows(None, [899, 32], 2)
    want = torch.empty_like(q)
    attend(c, r, q, "f16", want, "f16")
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        attend(c, r, q, "f16", out, "f16")
    side.synchronize()
    assert torch.equal(out, want)
    k, v = (torch.randn(2, 2, 64, device="cuda:0") for _ in "kv")
    ws = torch.zeros(hh.hh_kv4_attention_workspace(c.desc, r, 8), dtype=torch.uint8, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        append(c, r, k, v, "f32")
        attend(c, r, q, "f16", out, "f16", ws=ws)
    for i in range(4):
        # Other rows and places each time: the graph reads them where they are.
        k.normal_()
        v.normal_()
        keep[1].copy_(ints([700 + i, 20 + i]))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        append(c, r, k, v, "f32")
        attend(c, r, q, "f16", want, "f16")
        torch.cuda.synchronize()
        assert torch.equal(got, want), i


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB, its used pages at both ends."""
    hkv, n_pages = 8, 500_000  # 4.6 GB
    pool = torch.empty((n_pages, hkv, kv4.BLOCK), dtype=torch.uint8, device="cuda:0")
    table = ints([[n_pages - 1, 0, n_pages - 2]])
    desc = hh.hh_kv4_pool(pool.data_ptr(), table.data_ptr(), n_pages, hkv, 3, 1)
    c = Cache(1, hkv, 3)
    rng = np.random.default_rng(0)
    k, v = (rng.standard_normal((40, hkv, 64)).astype(np.float32) for _ in "kv")
    c.desc = desc
    r, keep = c.rows([0, 40], [0], 40)
    append(c, r, dev(k), dev(v), "f32")
    kb, vb = (torch.empty((40, hkv, 64), device="cuda:0") for _ in "kv")
    hh.hh_kv4_read(desc, r, kb.data_ptr(), vb.data_ptr(), hh.HH_F32, hkv * 64, hkv * 64, stream())
    assert np.array_equal(kb.cpu().numpy(), kv4.values(k).astype(np.float32))
    q = torch.randn(1, hkv, 64, device="cuda:0")
    out = torch.empty_like(q)
    r, keep = c.rows([0, 1], [39], 1)
    attend(c, r, q, "f32", out, "f32")
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), kv4.values(k), kv4.values(v), 0.125, 39, "f32")
