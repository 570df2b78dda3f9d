"""The 8-bit paged cache's operators on the GPU against the fp64 oracle.

* Appended bytes and values read back are exact (powers of two and whole numbers; keys
  are rotated in 64 bits and rounded once), and only the call's pages are written.
* Selected blocks are exact: scores are whole numbers times powers of two.
* Attention is compared with fp64 attention over the values that the pages hold.
  Its bound, for every element (a = max over the attended keys of
  scale * sum |q_i k_i|, m = max |v|):
    - scores: queries as two fp16 terms, 2^-22 of each product, and 64 fp32 sums, 2^-18 of
      sum |q k|; or, of few columns, as whole numbers, 2^-22 of the largest element each,
      64 of them 2^-16 max |q| max |k|, below 2^-18 max |k| sum |q| where the sum is over four
      times the largest, as of the N(0, 1) rows here (and none at all where elements are
      whole numbers of the scale); a rotation in fp32, 3 * 2^-24 more; the power's argument
      and the exponential, 2^-20 and 2^-21 of a weight (|argument| < 2^7):
      e = 2^-17.5 a + 2^-19;
    - weights relative to their sum: 2 e, and two fp16 terms each, 2 * 2^-22; sums of
      n weights and products in fp32: pairs of pages at 2^-24 each, n / 32 of them at
      most, here below 2^-17;
    - so |out - ref| <= m (2 e + 2^-21 + 2^-17) + half a step of the output's type.
* Pools start as 0xff bytes: scales and summaries of pages that nothing was appended to are
  NaN, and pages that no row may read would show.
"""
import numpy as np
import pytest

from oracle import kv4, kv8
from paper_2606_12154_amd import hh

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f32": (hh.HH_F32, torch.float32), "f16": (hh.HH_F16, torch.float16), "bf16": (hh.HH_BF16, torch.bfloat16)}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def dev(a, dtype=None):
    return torch.as_tensor(a, dtype=dtype, device="cuda:0")


def ints(a):
    return dev(np.asarray(a, dtype=np.int32))


def rope_table(n):
    ang = np.arange(n)[:, None] * 1e4 ** (-np.arange(32) / 32.0)
    return np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)


def stream():
    return torch.cuda.current_stream().cuda_stream


class Cache:
    """A pool of 0xff bytes with a shuffled page for every slot of the table, and the
    oracle's own."""

    def __init__(self, seqs, hkv, max_pages, seed=0, spare=3):
        self.hkv, self.max_pages, self.seqs = hkv, max_pages, seqs
        n = seqs * max_pages
        self.n_pages = n + spare
        self.table = np.random.default_rng(seed).permutation(self.n_pages)[:n].reshape(seqs, max_pages).astype(np.int32)
        self.pool = torch.full((self.n_pages, hkv, kv8.BLOCK), 255, dtype=torch.uint8, device="cuda:0")
        self.d_table = ints(self.table)
        self.desc = hh.hh_kv8_pool(self.pool.data_ptr(), self.d_table.data_ptr(), self.n_pages, hkv, max_pages, seqs)
        self.ref = kv8.Cache(seqs, max_pages, hkv)

    def rows(self, start, first, n_rows, table_row=None):
        keep = [None if a is None else ints(a) for a in (start, first, table_row)]
        longest = 1 if start is None else max(1, int(np.diff(start).max()))
        r = hh.hh_kv8_rows(*[None if t is None else t.data_ptr() for t in keep], len(first), n_rows, longest)
        return r, keep

    def append(self, lens, first, k, v, t, rope=None, ref=True):
        """Rows of sequences 0 .. of the cache, and of the oracle's."""
        start = np.concatenate([[0], np.cumsum(lens)])
        r, keep = self.rows(start, first, int(start[-1]))
        d_rope = None if rope is None else dev(rope)
        hh.hh_kv8_append(self.desc, r, k.data_ptr(), v.data_ptr(), TYPES[t][0], k.stride(0), v.stride(0),
                         None if rope is None else d_rope.data_ptr(), 0 if rope is None else len(rope), stream())
        torch.cuda.synchronize()
        if not ref:
            return
        kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
        for s, (n, f) in enumerate(zip(lens, first)):
            ks, vs = kf[start[s]:start[s + 1]], vf[start[s]:start[s + 1]]
            if rope is not None:
                pos = f + np.arange(n)
                ks = kv4.rotate(ks, rope, np.clip(pos, 0, len(rope) - 1)).astype(np.float32)
                n = min(n, len(rope) - f)
            self.ref.append(s, f, ks[:max(n, 0)], vs[:max(n, 0)])

    def check_bytes(self, touched):
        """Every block in `touched` ((sequence, page) pairs) as the oracle's, all others untouched."""
        got = self.pool.cpu().numpy()
        want = np.full((self.n_pages, self.hkv, kv8.BLOCK), 255, np.uint8)
        for s, p in touched:
            for h in range(self.hkv):
                want[self.table[s, p], h, :2128] = self.ref.blocks[s][p][h].bytes()
        for a, b in ((0, 1024), (1024, 2048), (2048, 2112), (2112, 2128), (2128, kv8.BLOCK)):
            assert np.array_equal(got[..., a:b], want[..., a:b]), (a, b, np.argwhere(got[..., a:b] != want[..., a:b])[:4])


def touched_by(lens, first, pages):
    return {(s, p) for s, (n, f) in enumerate(zip(lens, first)) for p in range(max(f, 0) // 16, pages)
            if n and max(f, 0) < min((p + 1) * 16, f + n) and f + n > p * 16}


def read(c, lens, first, t, table_row=None):
    n = sum(lens)
    r, keep = c.rows(np.concatenate([[0], np.cumsum(lens)]), first, n, table_row)
    back = [torch.full((n, c.hkv, 64), 9.0, dtype=TYPES[t][1], device="cuda:0") for _ in "kv"]
    hh.hh_kv8_read(c.desc, r, back[0].data_ptr(), back[1].data_ptr(), TYPES[t][0], c.hkv * 64, c.hkv * 64, stream())
    return back


def special(x):
    """Rows on the format's borders among ordinary ones [n, heads, 64]."""
    n = x.shape[0]
    for i, f in enumerate([lambda a: a * 0, lambda a: a * 1e-7, lambda a: a * 2.0 ** -15, lambda a: a * 3e4,
                           lambda a: np.where(np.arange(64) % 2, 127.0, 2.5 * np.sign(a)), lambda a: a * 1e-30]):
        if n > 2 * i:
            x[2 * i, i % x.shape[1]] = f(x[2 * i, i % x.shape[1]])
    return x


# ------------------------------------------------------------------ append and read

@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("lens,first", [([1], [0]), ([1, 1, 1], [0, 16, 32]), ([40, 3], [0, 16]), ([16, 1, 33], [48, 0, 16])])
def test_append_bytes_and_read(t, rope, lens, first):
    rng = np.random.default_rng(len(lens) + first[0])
    hkv, n = 3, sum(lens)
    c = Cache(len(lens), hkv, 4)
    wide = torch.zeros((n, 2 * hkv + 1, 64), dtype=TYPES[t][1], device="cuda:0")
    for i in range(2):
        wide[:, i * hkv:(i + 1) * hkv] = dev(special(rng.standard_normal((n, hkv, 64))), torch.float32).to(TYPES[t][1])
    c.append(lens, first, wide[:, :hkv], wide[:, hkv:2 * hkv], t, rope_table(64) if rope else None)
    c.check_bytes(touched_by(lens, first, 4))
    back = read(c, lens, first, t)
    for i in range(2):
        ref = np.concatenate([c.ref.values(s, f + m)[i][f:] for s, (m, f) in enumerate(zip(lens, first))])
        ref = torch.from_numpy(ref).to(TYPES[t][1])
        assert np.array_equal(back[i].double().cpu().numpy(), ref.double().numpy(), equal_nan=True)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("sizes", [(5, 1, 1, 1, 9, 4), (16, 15, 1, 2), (1,) * 18, (3, 40, 7), (31, 2, 17)])
def test_pages_that_fill_over_several_calls(t, rope, sizes):
    """Kept codes are requantized as scales grow; every state is the oracle's."""
    rng = np.random.default_rng(sum(sizes))
    c = Cache(2, 2, 5)
    first, done = 0, set()
    for i, n in enumerate(sizes):
        # The second sequence lags a slot behind; rows of sizes that differ by 2^12.
        lens, firsts = [n, n], [first, first]
        x = [rng.standard_normal((2 * n, 2, 64)) * np.exp2(rng.uniform(-8, 4, (2 * n, 2, 1))) for _ in "kv"]
        c.append(lens, firsts, *(dev(a, torch.float32).to(TYPES[t][1]) for a in x), t, rope_table(80) if rope else None)
        done |= touched_by(lens, firsts, 5)
        c.check_bytes(done)
        first += n


def test_cut_sequences_are_appended_to_at_their_new_end():
    rng = np.random.default_rng(5)
    c = Cache(1, 1, 4)

    def rows(n, size):
        return [dev(rng.standard_normal((n, 1, 64)) * size, torch.float32) for _ in "kv"]

    c.append([45], [0], *rows(45, 1.0), "f32")
    c.append([2], [19], *rows(2, 0.01), "f32")     # drops 21 .. 31, keeps the page's scale
    c.check_bytes({(0, 0), (0, 1), (0, 2)})
    c.append([1], [16], *rows(1, 0.01), "f32")     # a page's first slot: its scale anew
    c.append([40], [17], *rows(40, 30.0), "f32")
    c.check_bytes({(0, 0), (0, 1), (0, 2), (0, 3)})


@pytest.mark.parametrize("hkv", [3, 5, 8])
def test_many_rows_of_several_heads_a_workgroup(hkv):
    lens, first = [900, 1, 333, 33], [3, 40, 0, 15]
    c = Cache(4, hkv, 60)
    k, v = (torch.randn(sum(f for f in first), hkv, 64, device="cuda:0") for _ in "kv")
    c.append(first, [0] * 4, k, v, "f32")  # what they come behind
    k, v = (torch.randn(sum(lens), hkv, 64, device="cuda:0") for _ in "kv")
    c.append(lens, first, k, v, "f32")
    for got, i in zip(read(c, lens, first, "f32"), range(2)):
        want = np.concatenate([c.ref.values(s, f + m)[i][f:] for s, (m, f) in enumerate(zip(lens, first))])
        assert np.array_equal(got.double().cpu().numpy(), want)


def test_rows_that_are_not_finite():
    c = Cache(1, 2, 2)
    k, v = (torch.randn(20, 2, 64, device="cuda:0") for _ in "kv")
    k[3, 1, 40], v[7, 0, 1], v[8, 1, 63] = float("nan"), float("inf"), -float("inf")
    c.append([10], [0], k[:10], v[:10], "f32")
    c.append([10], [10], k[10:].contiguous(), v[10:].contiguous(), "f32")  # marks of kept slots stay
    c.check_bytes({(0, 0), (0, 1)})
    for got, bad in zip(read(c, [20], [0], "f32"), ([(3, 1)], [(7, 0), (8, 1)])):
        want = torch.zeros(20, 2, 64, dtype=torch.bool)
        for i, h in bad:
            want[i, h] = True
        assert torch.equal(torch.isnan(got.cpu()), want)
    c.append([1], [3], k[:1].contiguous(), v[:1].contiguous(), "f32")  # and go with the slots
    c.check_bytes({(0, 0), (0, 1)})
    assert torch.isfinite(read(c, [4], [0], "f32")[0]).all()


def test_padding_and_places_past_the_table():
    """Rows at negative positions and past the table or the rotation's are skipped
    by append and read as 0; a table row out of range has no page."""
    c = Cache(2, 1, 2)
    n = 10
    k, v = (torch.randn(n, 1, 64, device="cuda:0") for _ in "kv")
    # Sequences: 3 rows at -2, -1, 0; 3 rows at 30 .. 32 (the table ends at 32); one row of
    # table row 7, one of table row -1; none at 5; two at -9, -8.
    c.append([0, 30], [0, 0], *(torch.randn(30, 1, 64, device="cuda:0") for _ in "kv"), "f32")
    start, first, trow = [0, 3, 6, 7, 8, 8, 10], [-2, 30, 0, 0, 5, -9], [0, 1, 7, -1, 0, 0]
    r, keep = c.rows(start, first, n, table_row=trow)
    hh.hh_kv8_append(c.desc, r, k.data_ptr(), v.data_ptr(), hh.HH_F32, 64, 64, None, 0, stream())
    c.ref.append(0, -2, k[:3].cpu().numpy(), v[:3].cpu().numpy())
    c.ref.append(1, 30, k[3:6].cpu().numpy(), v[3:6].cpu().numpy())
    c.check_bytes({(0, 0), (1, 0), (1, 1)})
    kb, vb = (torch.full((n, 1, 64), 5.0, device="cuda:0") for _ in "kv")
    hh.hh_kv8_read(c.desc, r, kb.data_ptr(), vb.data_ptr(), hh.HH_F32, 64, 64, stream())
    for i, got in enumerate((kb, vb)):
        want = np.zeros((n, 1, 64))
        want[2], want[3:5] = c.ref.values(0, 1)[i][0], c.ref.values(1, 32)[i][30:]
        assert np.array_equal(got.double().cpu().numpy(), want)
    # A rotation table that ends before the rows: those are skipped.
    c2 = Cache(1, 1, 2)
    c2.append([10], [0], k, v, "f32", rope_table(4))
    c2.check_bytes({(0, 0)})
    back = read(c2, [10], [0], "f32")
    assert (back[0][4:] == 0).all() and (back[0][:4] != 0).any()


# ------------------------------------------------------------------ attention

def filled(lens, hkv, seed, max_pages=None):
    """A cache that holds lens[i] positions of sequence i."""
    rng = np.random.default_rng(seed)
    c = Cache(len(lens), hkv, max_pages or max(1, (max(lens) + 15) // 16), seed)
    x = [rng.standard_normal((sum(lens), hkv, 64)).astype(np.float32) for _ in "kv"]
    if sum(lens):
        c.append(lens, [0] * len(lens), dev(x[0]), dev(x[1]), "f32")
    return c, rng


def bound(q, k, v, scale, ot):
    a = scale * np.abs(q).sum(-1).max() * np.abs(k).max() if len(k) else 0.0
    e = 2.0 ** -17.5 * a + 2.0 ** -19
    return np.abs(v).max(initial=0.0) * (2 * e + 2.0 ** -21 + 2.0 ** -17), HALF_STEP[ot]


def attend(c, r, q, t, out, ot, scale=0.125, rope=None, blocks=None, ws=None):
    """Attention over all keys, or over a device list of blocks."""
    hq, d_rope = q.shape[1], None if rope is None else dev(rope)
    n = 0 if blocks is None else blocks.shape[-1]
    need = (hh.hh_kv8_attention_workspace(c.desc, r, hq) if blocks is None
            else hh.hh_kv8_attention_blocks_workspace(c.desc, r, hq, n))
    if ws is None:
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda:0")
    args = (q.data_ptr(), TYPES[t][0], q.stride(0), hq, scale, None if rope is None else d_rope.data_ptr(),
            0 if rope is None else len(rope), out.data_ptr(), TYPES[ot][0], out.stride(0), ws.data_ptr() if need else None,
            ws.numel(), stream())
    if blocks is None:
        hh.hh_kv8_attention(c.desc, r, *args)
    else:
        hh.hh_kv8_attention_blocks(c.desc, r, blocks.data_ptr(), n, *args)
    torch.cuda.synchronize()
    return ws


def listed_reference(q, k, v, scale, first, lists, hkv):
    """fp64 attention of rows q [n, heads, 64] over the blocks in lists [n, hkv, m]."""
    out, group = np.zeros_like(q), q.shape[1] // hkv
    for i in range(len(q)):
        pos = first + i
        for h in range(hkv):
            at = [b * 16 + np.arange(16) for b in lists[i, h] if 0 <= b <= pos // 16 and pos >= 0]
            at = np.concatenate(at) if at else np.zeros(0, int)
            at = at[at <= pos]
            at = at[at < len(k)]
            if not len(at):
                continue
            s = q[i, h * group:(h + 1) * group] @ k[at, h].T * scale
            with np.errstate(invalid="ignore"):
                w = np.exp(s - s.max(-1, keepdims=True))
                out[i, h * group:(h + 1) * group] = w @ v[at, h] / w.sum(-1, keepdims=True)
    return out


def check(c, lens, first, hq, t, ot, rng, rope=None, scale=0.125, lists=None):
    """Rows lens[i] at first[i] of each sequence, with everything around them checked."""
    n = sum(lens)
    start = np.concatenate([[0], np.cumsum(lens)])
    r, keep = c.rows(start, first, n + 2)  # two rows of no sequence
    q = dev(rng.standard_normal((n + 2, hq, 64)), torch.float32).to(TYPES[t][1])
    out = torch.full((n + 2, hq + 1, 64), 7.0, dtype=TYPES[ot][1], device="cuda:0")[:, :hq]
    d_lists = None if lists is None else ints(lists)
    attend(c, r, q, t, out, ot, scale, rope, d_lists)
    got, qf = out.double().cpu().numpy(), q.double().cpu().numpy()
    assert (got[n:] == 7.0).all(), "rows of no sequence"
    for s in range(len(lens)):
        rows = qf[start[s]:start[s + 1]]
        if not len(rows):
            continue
        pos = first[s] + np.arange(len(rows))
        if rope is not None:
            rows = kv4.rotate(rows, rope, np.clip(pos, 0, len(rope) - 1))
        k, v = c.ref.values(s, min(max(int(pos[-1]) + 1, 0), c.max_pages * 16))
        if lists is None:
            want = kv4.attend(rows, k, v, scale, first[s])
        else:
            want = listed_reference(rows, k, v, scale, first[s], lists[start[s]:start[s + 1]], c.hkv)
        e, half = bound(rows, k, v, scale, ot)
        err = np.abs(got[start[s]:start[s + 1]] - want)
        assert (err <= e + half * (np.abs(want) + e)).all(), (s, err.max(), e)
    return got


SHAPES = [([1], [0]), ([1], [299]), ([1, 1, 1, 1], [0, 15, 16, 77]), ([5], [0]), ([3, 1, 40], [14, 200, 0]), ([70], [33]),
          ([1, 2], [700, 1500]), ([130, 9], [0, 250])]


@pytest.mark.parametrize("t,ot,rope", [("f32", "f32", False), ("f32", "bf16", True), ("f16", "f16", False), ("bf16", "f32", True),
                                       ("bf16", "bf16", False)])
@pytest.mark.parametrize("lens,first", SHAPES)
def test_attention(t, ot, rope, lens, first):
    c, rng = filled([n + f for n, f in zip(lens, first)], 2, len(lens) + first[0])
    check(c, lens, first, 8, t, ot, rng, rope_table(2048) if rope else None)


@pytest.mark.parametrize("hkv,group", [(1, 1), (3, 1), (2, 3), (1, 7), (2, 8), (1, 12), (1, 16), (1, 40)])
@pytest.mark.parametrize("lens,first", [([1, 1], [20, 130]), ([19], [40])])
def test_attention_head_layouts(hkv, group, lens, first):
    c, rng = filled([n + f for n, f in zip(lens, first)], hkv, group)
    check(c, lens, first, hkv * group, "f32", "f32", rng)


@pytest.mark.parametrize("scale", [1e-30, 1.0, 4.0])
def test_attention_scales(scale):
    c, rng = filled([150], 1, 3)
    check(c, [4], [146], 4, "f32", "f32", rng, scale=scale)


def test_padding_rows_and_empty_sequences():
    c, rng = filled([40, 40, 40], 2, 9)
    got = check(c, [3, 0, 2], [-2, 7, -5], 4, "f32", "f32", rng)
    assert (got[:2] == 0).all() and (got[2] != 0).any() and (got[3:5] == 0).all()


def test_positions_past_the_table_see_all_of_it():
    c, rng = filled([32], 1, 4)
    q = torch.randn(2, 2, 64, device="cuda:0")
    out = torch.empty_like(q)
    for at in (40, 1 << 29, (1 << 31) - 5):
        r, keep = c.rows([0, 2], [at], 2)
        attend(c, r, q, "f32", out, "f32")
        k, v = c.ref.values(0, 32)
        want = kv4.attend(q.double().cpu().numpy(), k, v, 0.125, 31)
        want[1] = kv4.attend(q[1:].double().cpu().numpy(), k, v, 0.125, 31)[0]
        assert np.abs(out.double().cpu().numpy() - want).max() < 1e-4


@pytest.mark.parametrize("lens,first,hkv,group", [([1], [5000], 2, 4), ([2, 1], [4001, 90], 1, 8), ([20], [6000], 1, 4)])
def test_split_ranges(lens, first, hkv, group):
    c, rng = filled([n + f for n, f in zip(lens, first)], hkv, 6)
    r, keep = c.rows(np.concatenate([[0], np.cumsum(lens)]), first, sum(lens))
    assert hh.hh_kv8_attention_workspace(c.desc, r, hkv * group) > 0
    check(c, lens, first, hkv * group, "f32", "f32", rng)


@pytest.mark.parametrize("lens,first", [([16], [0]), ([1], [300]), ([40], [280])])
def test_what_is_not_finite_reaches_the_rows_that_see_it(lens, first):
    c, rng = filled([lens[0] + first[0]], 2, 8)
    n = lens[0] + first[0]
    bad_k, bad_v = n - 1 - (n - 1) % 3, max(n - 9, 0)
    k, v = (torch.randn(n, 2, 64, device="cuda:0") for _ in "kv")
    k[bad_k, 0, 3], v[bad_v, 1, 60] = float("inf"), float("nan")
    c.append([n], [0], k, v, "f32")
    r, keep = c.rows([0, lens[0]], first, lens[0])
    q = torch.randn(lens[0], 8, 64, device="cuda:0")
    out = torch.empty_like(q)
    attend(c, r, q, "f32", out, "f32")
    nan = torch.isnan(out).cpu().numpy()
    pos = first[0] + np.arange(lens[0])
    assert (nan[:, :4] == (pos >= bad_k)[:, None, None]).all() and (nan[:, 4:] == (pos >= bad_v)[:, None, None]).all()


def test_queries_that_are_not_finite():
    c, rng = filled([100], 1, 8)
    q = torch.randn(3, 4, 64, device="cuda:0")
    q[1, 2, 5] = float("nan")
    r, keep = c.rows([0, 3], [97], 3)
    out = torch.empty_like(q)
    attend(c, r, q, "f32", out, "f32")
    nan = torch.isnan(out).cpu()
    want = torch.zeros_like(nan)
    want[1, 2] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("t,top", [("f32", 2.0 ** 127), ("bf16", 2.0 ** 127), ("f16", 2.0 ** 15)])
@pytest.mark.parametrize("rows", [1, 20])
@pytest.mark.parametrize("listed", [False, True])
def test_scores_past_fp32(t, top, rows, listed):
    """scale * q . k above 2^128: the largest score takes all, and keys that a query does not
    see (a product of 0) count alike.  One weight of 1, or 40 equal ones in two fp16
    terms: 2^-22 each and in their sum, and 40 sums of 2^-24."""
    scale, n, rng = 2.0 ** 100, 40, np.random.default_rng(2)
    for seen in (True, False):
        k = np.zeros((n, 1, 64), np.float32)
        k[:, 0, 0 if seen else 1] = 7 * np.arange(n) % n - 20  # (exact in the cache, no two alike)
        v = rng.standard_normal((n, 1, 64)).astype(np.float32)
        c = Cache(1, 1, 3)
        c.append([n], [0], dev(k), dev(v), "f32")
        q = np.zeros((rows, 4, 64), np.float32)
        q[:, :, 0] = top
        r, keep = c.rows([0, rows], [n - rows], rows)
        out = torch.empty(rows, 4, 64, device="cuda:0")
        blocks = dev(np.tile(np.arange(3, dtype=np.int32), (rows, 1, 1))) if listed else None
        attend(c, r, dev(q).to(TYPES[t][1]), t, out, "f32", scale, blocks=blocks)
        kk, vv = c.ref.values(0, n)
        want = kv4.attend(q.astype(np.float64), kk, vv, scale, n - rows)
        assert np.isfinite(want).all()
        err = np.abs(out.double().cpu().numpy() - want)
        assert (err <= np.abs(vv).max() * (2 * 2.0 ** -22 + 40 * 2.0 ** -24 + 2.0 ** -24)).all(), (seen, err.max())


def test_weights_far_apart():
    """One key takes nearly all of the weight and has a small value; the many others'
    weights of about 2^-20 make the sum of its other dimensions."""
    n = 4000
    k, v = np.zeros((n, 1, 64), np.float32), np.zeros((n, 1, 64), np.float32)
    k[:, 0, 1] = np.random.default_rng(0).standard_normal(n) * 0.1
    k[100, 0, 0] = 64.0
    v[:, 0, 1:] = 1.0
    v[100, 0] = 0.0
    c = Cache(1, 1, 250)
    c.append([n], [0], dev(k), dev(v), "f32")
    q = np.zeros((1, 1, 64), np.float32)
    q[0, 0, 0], q[0, 0, 1] = 1.75, 1.0
    out = torch.empty(1, 1, 64, device="cuda:0")
    r, keep = c.rows([0, 1], [n - 1], 1)
    attend(c, r, dev(q), "f32", out, "f32")
    want = kv4.attend(q, *c.ref.values(0, n), 0.125, n - 1)
    # Weights relative to 2^-22, sums of 4,000 in fp32 (125 pairs of pages: 2^-17), and the
    # scores' 2^-17.5 of 14 and 2^-19, which move the largest against the others.
    assert 0 < want[0, 0, 5] < 1e-2
    assert np.abs(out.double().cpu().numpy() / np.maximum(want, 1e-300) - 1)[0, 0, 1:].max() < 2 * (14 * 2.0 ** -17.5 + 2.0 ** -19) + 2.0 ** -16


# ------------------------------------------------------------------ listed blocks

def random_lists(lens, first, hkv, n, rng):
    """Blocks in any order, with entries that are none."""
    out = np.full((sum(lens), hkv, n), -1, np.int32)
    pos = np.concatenate([f + np.arange(m) for f, m in zip(first, lens)])
    for i, p in enumerate(pos):
        for h in range(hkv):
            if p >= 0:
                some = rng.permutation(p // 16 + 1)[:n]
                some = some[:max(1, len(some) - int(rng.integers(0, 2)))]
                out[i, h, rng.permutation(n)[:len(some)]] = some
    return out


@pytest.mark.parametrize("t,ot,rope", [("f32", "f32", False), ("f16", "f16", False), ("bf16", "f32", True)])
@pytest.mark.parametrize("lens,first", SHAPES)
@pytest.mark.parametrize("n", [1, 2, 5, 40])
def test_listed_blocks(t, ot, rope, lens, first, n):
    c, rng = filled([m + f for m, f in zip(lens, first)], 2, len(lens) + first[0])
    lists = np.concatenate([random_lists(lens, first, 2, n, rng), np.full((2, 2, n), 0, np.int32)])
    check(c, lens, first, 8, t, ot, rng, rope_table(2048) if rope else None, lists=lists)


@pytest.mark.parametrize("rows,n,group", [(1, 9, 4), (1, 300, 4), (40, 25, 4), (300, 8, 2), (700, 6, 4), (700, 6, 16), (2500, 3, 1)])
def test_listed_blocks_every_way_of_cutting(rows, n, group):
    """Few rows and many: one to eight waves a row, split lists; 16-bit types."""
    c, rng = filled([3000], 2, rows)
    lists = np.concatenate([random_lists([rows], [3000 - rows], 2, n, rng), np.zeros((2, 2, n), np.int32)])
    for t in ("f32", "f16"):
        check(c, [rows], [3000 - rows], 2 * group, t, t, rng, lists=lists)


@pytest.mark.parametrize("hkv,group", [(1, 1), (3, 2), (1, 8), (2, 12), (1, 16), (1, 40)])
def test_listed_blocks_head_layouts(hkv, group):
    lens, first = [1, 6], [333, 100]
    c, rng = filled([m + f for m, f in zip(lens, first)], hkv, group)
    lists = np.concatenate([random_lists(lens, first, hkv, 7, rng), np.zeros((2, hkv, 7), np.int32)])
    check(c, lens, first, hkv * group, "f32", "f32", rng, lists=lists)


def test_lists_of_every_kind():
    """Empty ones, entries out of range, one twice, a lone last block; padding rows."""
    lens, first = [6, 2], [90, -1]
    c, rng = filled([96, 5], 1, 2)
    lists = np.array([[-1] * 6, [6, -7, 99, 1 << 30, -(1 << 31), 6], [2, 2, -1, 3, -1, 2], [5, -1, -1, -1, -1, -1],
                      [-1, -1, -1, -1, -1, 0], [5, 4, 3, 2, 1, 0], [0, 0, 0, 0, 0, 0], [0, 1, 2, 3, 4, 5], [0] * 6, [0] * 6],
                     np.int64).astype(np.int32)[:, None]
    got = check(c, lens, first, 4, "f32", "f32", rng, lists=lists)
    assert (got[:2] == 0).all() and (got[6] == 0).all() and (got[2:6] != 0).any((1, 2)).all() and (got[7] != 0).any()


@pytest.mark.parametrize("n", [300, 301, 1500])
def test_long_lists(n):
    """Lists that are split over workgroups, and over more steps than a wave holds at once."""
    c, rng = filled([16 * 1600], 1, 1)
    lists = np.stack([rng.permutation(1600)[:n] for _ in range(3)])[:, None].astype(np.int32)
    lists[:, :, 70:200] = -1
    lists[1] = -1
    lists[1, :, -1] = 5
    check(c, [1], [16 * 1600 - 1], 4, "f32", "f32", rng, lists=lists)


@pytest.mark.parametrize("group", [4, 12])
def test_entries_that_are_none_read_no_page(group):
    """A sequence whose first pages were never written (bytes that make NaN scales), and
    lists of its others with entries that are none beside them."""
    rng = np.random.default_rng(0)
    c = Cache(1, 1, 6)
    k, v = (torch.randn(64, 1, 64, device="cuda:0") for _ in "kv")
    c.append([64], [32], k, v, "f32")
    lists = np.array([[2, -1, -1, 3, 5, -1, -1, -1], [-1, -1, 4, -1, -1, 99, 2, -1]], np.int32)[:, None]
    lists = np.concatenate([lists, np.zeros((2, 1, 8), np.int32)])
    check(c, [2], [93], group, "f32", "f32", rng, lists=lists)


@pytest.mark.parametrize("group", [4, 12])
def test_lists_whose_scores_are_all_low(group):
    """Scores far below 0, of blocks that stand beside entries that are none: their
    weights go by the largest of them, in whatever order the blocks come."""
    n = 16 * 140
    c = Cache(1, 1, 140)
    k, v = (torch.randn(n, 1, 64, device="cuda:0") for _ in "kv")
    k[:, :, 0] = 60.0
    c.append([n], [0], k, v, "f32")
    lists = np.full((3, 1, 140), -1, np.int32)
    lists[0, 0, [1, 8, 133]] = [139, 5, 7]   # (the right side's first blocks come last)
    lists[1, 0, 138] = 139
    lists[2, 0, [0, 3, 64, 139]] = [139, 2, 3, 4]
    q = torch.randn(3, group, 64, device="cuda:0")
    q[:, :, 0] = -50.0
    out = torch.empty_like(q)
    for i in range(3):
        r, keep = c.rows([0, 1], [n - 1], 1)
        one = out[i:i + 1]
        attend(c, r, q[i:i + 1].contiguous(), "f32", one, "f32", blocks=ints(lists[i:i + 1]))
        kk, vv = c.ref.values(0, n)
        rows = q[i:i + 1].double().cpu().numpy()
        want = listed_reference(rows, kk, vv, 0.125, n - 1, lists[i:i + 1], 1)
        e, half = bound(rows, kk, vv, 0.125, "f32")
        assert (np.abs(one.double().cpu().numpy() - want) <= e + half * (np.abs(want) + e)).all()


def test_a_list_of_all_blocks_is_the_attention_over_all_keys():
    c, rng = filled([700], 2, 3)
    lists = np.full((5, 2, 44), -1, np.int32)
    lists[:, :] = np.arange(44)
    q = torch.randn(3, 8, 64, device="cuda:0")
    out = [torch.empty_like(q) for _ in "ab"]
    r, keep = c.rows([0, 3], [697], 3)
    attend(c, r, q, "f32", out[0], "f32")
    attend(c, r, q, "f32", out[1], "f32", blocks=ints(lists[:3]))
    assert torch.allclose(out[0], out[1], atol=1e-5, rtol=0)


def test_marked_slots_of_listed_blocks():
    """NaN reaches the rows that list its block and see its slot, alone."""
    c = Cache(1, 1, 8)
    k, v = (torch.randn(120, 1, 64, device="cuda:0") for _ in "kv")
    k[37, 0, 0] = float("nan")
    c.append([120], [0], k, v, "f32")
    lists = np.full((20, 1, 3), -1, np.int32)
    lists[:, 0, 0] = np.where(np.arange(20) % 2, 2, 1)
    lists[:, 0, 2] = 0
    q = torch.randn(20, 2, 64, device="cuda:0")
    out = torch.empty_like(q)
    r, keep = c.rows([0, 20], [30], 20)
    attend(c, r, q, "f32", out, "f32", blocks=ints(lists))
    want = (np.arange(20) % 2 == 1) & (30 + np.arange(20) >= 37)
    assert (torch.isnan(out).cpu().numpy() == want[:, None, None]).all()


# ------------------------------------------------------------------ selection

def select(c, r, q, t, n, first, last, rope=None, out=None):
    need = hh.hh_kv8_select_workspace(c.desc, r, q.shape[1], n)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda:0")
    d_rope = None if rope is None else dev(rope)
    if out is None:
        out = torch.full((q.shape[0], c.hkv, n), -7, dtype=torch.int32, device="cuda:0")
    hh.hh_kv8_select(c.desc, r, q.data_ptr(), TYPES[t][0], q.stride(0), q.shape[1], None if rope is None else d_rope.data_ptr(),
                     0 if rope is None else len(rope), n, first, last, out.data_ptr(), ws.data_ptr() if need else None, need, stream())
    torch.cuda.synchronize()
    return out


def check_selection(c, lens, first, hq, t, n, keep_first, keep_last, rng, rope=None, q=None):
    m, start = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    r, keep = c.rows(start, first, m + 1)
    if q is None:
        q = dev(rng.standard_normal((m + 1, hq, 64)), torch.float32).to(TYPES[t][1])
    got = select(c, r, q, t, n, keep_first, keep_last, rope).cpu().numpy()
    assert (got[m:] == -7).all(), "rows of no sequence"
    qf, group = q.double().cpu().numpy(), hq // c.hkv
    for s in range(len(lens)):
        for i in range(lens[s]):
            pos, row = first[s] + i, start[s] + i
            x = qf[row:row + 1]
            if rope is not None:
                x = kv4.rotate(x, rope, np.clip([pos], 0, len(rope) - 1))
            for h in range(c.hkv):
                want = kv8.select(x[0, h * group:(h + 1) * group], [p[h] for p in c.ref.blocks[s]], pos, n, keep_first, keep_last)
                assert np.array_equal(got[row, h], want), (s, i, h, got[row, h], want)
    return got


@pytest.mark.parametrize("t,rope", [("f32", False), ("f32", True), ("f16", True), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("lens,first", [([1], [0]), ([1, 1], [700, 90]), ([3, 20], [300, 111]), ([2, 0, 1], [-1, 5, 800])])
@pytest.mark.parametrize("n,keep_first,keep_last", [(1, 0, 1), (6, 1, 2), (9, 0, 4), (16, 2, 14), (60, 1, 1)])
def test_selection(t, rope, lens, first, n, keep_first, keep_last):
    c, rng = filled([max(m + f, 0) for m, f in zip(lens, first)], 2, first[0] + 5)
    check_selection(c, lens, first, 8, t, n, keep_first, keep_last, rng, rope_table(1024) if rope else None)


@pytest.mark.parametrize("t,rope", [("f32", True), ("f16", False), ("bf16", True)])
@pytest.mark.parametrize("lens,first,n,keep_first,keep_last", [
    ([8, 33, 0, 17], [300, 77, 4, 0], 5, 1, 2), ([50], [0], 3, 0, 1), ([40, 9], [-3, 390], 6, 2, 4), ([20], [470], 29, 0, 1)])
def test_selection_of_rows_together(t, rope, lens, first, n, keep_first, keep_last):
    """Rows that take all of their blocks beside rows that do not, in one tile."""
    c, rng = filled([max(m + f, 0) for m, f in zip(lens, first)], 2, 3)
    check_selection(c, lens, first, 6, t, n, keep_first, keep_last, rng, rope_table(1024) if rope else None)


@pytest.mark.parametrize("hkv,group", [(1, 1), (3, 1), (1, 5), (2, 16), (1, 40)])
def test_selection_head_layouts(hkv, group):
    c, rng = filled([500, 120], hkv, 2)
    check_selection(c, [1, 2], [499, 118], hkv * group, "f32", 5, 1, 1, rng)


@pytest.mark.parametrize("rows", [1, 20])
def test_equal_scores_go_to_the_lowest_blocks(rows):
    c = Cache(1, 1, 40)
    k = torch.randn(16, 1, 64, device="cuda:0").repeat(40, 1, 1)
    k[16 * 20:16 * 21] *= 3
    c.append([640], [0], k, k, "f32")
    rng = np.random.default_rng(0)
    got = check_selection(c, [rows], [640 - rows], 1, "f32", 8, 2, 3, rng)
    assert got[rows - 1, 0].tolist() in ([0, 1, 2, 3, 20, 37, 38, 39], [0, 1, 2, 3, 4, 37, 38, 39])
    for x in (0.0, float("inf"), float("nan")):
        q = torch.full((rows + 1, 1, 64), x, device="cuda:0")
        got = check_selection(c, [rows], [640 - rows], 1, "f32", 8, 2, 3, rng, q=q)
        assert got[rows - 1, 0].tolist() == [0, 1, 2, 3, 4, 37, 38, 39]


@pytest.mark.parametrize("rows", [1, 30])
def test_selection_over_scales_far_apart(rows):
    """Blocks whose scales differ by 2^20; huge and tiny queries."""
    rng = np.random.default_rng(4)
    c = Cache(1, 2, 30)
    k = rng.standard_normal((480, 2, 64)) * np.repeat(np.exp2(rng.uniform(-15, 12, (30, 2, 1))), 16, 0)
    c.append([480], [0], dev(k, torch.float32), dev(k, torch.float32), "f32")
    for size in (1e-30, 1.0, 1e30):
        q = dev(rng.standard_normal((rows + 1, 4, 64)) * size, torch.float32)
        check_selection(c, [rows], [480 - rows], 4, "f32", 7, 0, 1, rng, q=q)


@pytest.mark.parametrize("pages,rows", [(130, 1), (1100, 1), (1100, 300), (4200, 2), (9000, 1), (17000, 1), (500, 40), (250, 19),
                                        (100, 100), (4100, 700)])
def test_selection_over_many_blocks(pages, rows):
    """Every way of cutting the call up, against a sorted list of exact scores."""
    rng = np.random.default_rng(pages + rows)
    hkv, n, f, l = 2, 37, 1, 3
    c = Cache(1, hkv, pages)
    k = (rng.standard_normal((pages * 16, hkv, 64)) + np.repeat(rng.standard_normal((pages, hkv, 64)), 16, 0)).astype(np.float32)
    c.append([pages * 16], [0], dev(k), dev(k), "f32", ref=False)
    first = pages * 16 - rows
    r, keep = c.rows([0, rows], [first], rows)
    q = dev(rng.standard_normal((rows, hkv, 64)), torch.float32)
    got = select(c, r, q, "f32", n, f, l).cpu().numpy()
    raw = c.pool.cpu().numpy()[c.table[0]]  # [pages, hkv, 2176]
    m = raw[..., 2048:2112].copy().view(np.int8).astype(np.int64)
    scale = raw[..., 2112:2128].copy().view(np.float16)[..., 4].astype(np.float64)
    qf = q.double().cpu().numpy()
    for i in range(rows):
        nb = (first + i) // 16 + 1
        for h in range(hkv):
            score = (m[:, h] @ kv8.query_codes(qf[i, h:h + 1])) * scale[:, h]
            order = np.argsort(-score[f:nb - l], kind="stable")[:n - f - l] + f
            want = np.concatenate([np.arange(f), np.sort(order), np.arange(nb - l, nb)])
            assert np.array_equal(got[i, h], want), (i, h)


# ------------------------------------------------------------------ together

def test_a_stream_that_selects_what_it_reads():
    """Append, select and attend step by step, as a decoder would, from two graphs' worth
    of calls on their own stream; every step against the oracle."""
    rng = np.random.default_rng(12)
    hkv, hq, n = 2, 8, 5
    c = Cache(2, hkv, 20)
    lens, tab = [150, 97], rope_table(512)
    x = [rng.standard_normal((sum(lens), hkv, 64)).astype(np.float32) for _ in "kv"]
    c.append(lens, [0, 0], dev(x[0]), dev(x[1]), "f32", tab)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for step in range(20):
            pos = [m + step for m in lens]
            k, v = (dev(rng.standard_normal((2, hkv, 64)), torch.float32) for _ in "kv")
            c.append([1, 1], pos, k, v, "f32", tab)
            q = dev(rng.standard_normal((2, hq, 64)), torch.float32)
            r, keep = c.rows(None, pos, 2)
            blocks = select(c, r, q, "f32", n, 1, 2, tab)
            out = torch.empty_like(q)
            attend(c, r, q, "f32", out, "f32", rope=tab, blocks=blocks)
            got, lists, qf = out.double().cpu().numpy(), blocks.cpu().numpy(), q.double().cpu().numpy()
            for s in range(2):
                rows = kv4.rotate(qf[s:s + 1], tab, [pos[s]])
                for h in range(hkv):
                    assert np.array_equal(lists[s, h], kv8.select(rows[0, 4 * h:4 * h + 4], [p[h] for p in c.ref.blocks[s]], pos[s], n, 1, 2))
                kk, vv = c.ref.values(s, pos[s] + 1)
                want = listed_reference(rows, kk, vv, 0.125, pos[s], lists[s:s + 1], hkv)
                e, half = bound(rows, kk, vv, 0.125, "f32")
                assert (np.abs(got[s:s + 1] - want) <= e + half * (np.abs(want) + e)).all()


def test_captured_calls_replay():
    """Two graphs of append, select and attention over blocks on one pool, with
    workspaces of their own, replayed in turn with eager work between."""
    rng = np.random.default_rng(3)
    hkv, hq, n = 2, 8, 80
    c = Cache(2, hkv, 300)
    past = [4500, 3000]
    x = [rng.standard_normal((sum(past), hkv, 64)).astype(np.float32) for _ in "kv"]
    c.append(past, [0, 0], dev(x[0]), dev(x[1]), "f32", ref=False)
    first = ints(past)
    r = hh.hh_kv8_rows(None, first.data_ptr(), None, 2, 2, 1)

    class Step:
        def __init__(self):
            self.k, self.v = (torch.zeros(2, hkv, 64, device="cuda:0") for _ in "kv")
            self.q, self.out, self.all = (torch.zeros(2, hq, 64, device="cuda:0") for _ in "qoa")
            self.blocks = torch.zeros(2, hkv, n, dtype=torch.int32, device="cuda:0")
            sizes = (hh.hh_kv8_select_workspace(c.desc, r, hq, n), hh.hh_kv8_attention_blocks_workspace(c.desc, r, hq, n),
                     hh.hh_kv8_attention_workspace(c.desc, r, hq))
            self.ws = [torch.full((max(b, 1),), 255, dtype=torch.uint8, device="cuda:0") for b in sizes]

        def run(self):
            s, ws = stream(), self.ws
            hh.hh_kv8_append(c.desc, r, self.k.data_ptr(), self.v.data_ptr(), hh.HH_F32, hkv * 64, hkv * 64, None, 0, s)
            hh.hh_kv8_select(c.desc, r, self.q.data_ptr(), hh.HH_F32, hq * 64, hq, None, 0, n, 1, 2, self.blocks.data_ptr(),
                             ws[0].data_ptr(), ws[0].numel(), s)
            hh.hh_kv8_attention_blocks(c.desc, r, self.blocks.data_ptr(), n, self.q.data_ptr(), hh.HH_F32, hq * 64, hq, 0.125, None,
                                       0, self.out.data_ptr(), hh.HH_F32, hq * 64, ws[1].data_ptr(), ws[1].numel(), s)
            hh.hh_kv8_attention(c.desc, r, self.q.data_ptr(), hh.HH_F32, hq * 64, hq, 0.125, None, 0, self.all.data_ptr(),
                                hh.HH_F32, hq * 64, ws[2].data_ptr(), ws[2].numel(), s)

    steps = [Step(), Step()]
    graphs = []
    for st in steps:
        st.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    eager = Step()
    for turn in range(6):
        st, g = steps[turn % 2], graphs[turn % 2]
        first += 1
        for a in (st.k, st.v, st.q):
            a.normal_()
        before = c.pool.clone()
        g.replay()
        torch.cuda.synchronize()
        after = c.pool.clone()
        c.pool.copy_(before)
        for a, b in ((eager.k, st.k), (eager.v, st.v), (eager.q, st.q)):
            a.copy_(b)
        eager.run()
        torch.cuda.synchronize()
        assert torch.equal(c.pool, after) and torch.equal(eager.blocks, st.blocks)
        assert torch.equal(eager.out, st.out) and torch.equal(eager.all, st.all)


def test_equal_calls_give_equal_bits():
    c, rng = filled([3000, 2000], 4, 5)
    q = torch.randn(2, 16, 64, device="cuda:0").bfloat16()
    r, keep = c.rows(None, [2999, 1999], 2)
    outs = []
    for fill in (0, 255, 63):
        out = torch.empty_like(q)
        need = hh.hh_kv8_attention_workspace(c.desc, r, 16)
        attend(c, r, q, "bf16", out, "bf16", ws=torch.full((need,), fill, dtype=torch.uint8, device="cuda:0"))
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ------------------------------------------------------------------ the same calls elsewhere
#
# Results are compared bit by bit with those of calls that the tests above hold against the
# oracle: neither where a page or row lies nor what runs beside a call changes a result.

def every_call(c, r, q, t, n=6):
    """Attention over all keys, selection, and attention over what it selected."""
    out = [torch.full(q.shape, 7.0, dtype=TYPES[t][1], device="cuda:0") for _ in "ab"]
    attend(c, r, q, t, out[0], t)
    blocks = select(c, r, q, t, n, 1, 2)
    attend(c, r, q, t, out[1], t, blocks=blocks)
    return out[0], blocks, out[1]


@pytest.mark.parametrize("lens,first", [([1, 1], [299, 500]), ([70], [430])])
def test_pools_past_32_bits_of_bytes(lens, first):
    hkv, past = 2, [m + f for m, f in zip(lens, first)]
    c, rng = filled(past, hkv, 8)
    low = (1 << 32) // (hkv * kv8.BLOCK) + 1  # pages below the ones in use
    assert low * hkv * kv8.BLOCK > 1 << 32
    big = Cache(len(lens), hkv, c.max_pages, 8)
    big.pool = torch.full((low + c.n_pages, hkv, kv8.BLOCK), 255, dtype=torch.uint8, device="cuda:0")
    big.d_table = ints(big.table + low)
    big.desc = hh.hh_kv8_pool(big.pool.data_ptr(), big.d_table.data_ptr(), low + c.n_pages, hkv, c.max_pages, len(lens))
    again = np.random.default_rng(8)
    x = [again.standard_normal((sum(past), hkv, 64)).astype(np.float32) for _ in "kv"]
    big.append(past, [0] * len(past), dev(x[0]), dev(x[1]), "f32", ref=False)
    assert torch.equal(big.pool[low:], c.pool)
    assert (big.pool[:c.n_pages] == 255).all() and (big.pool[low - c.n_pages:low] == 255).all()
    for a, b in zip(read(c, past, [0] * len(past), "f32"), read(big, past, [0] * len(past), "f32")):
        assert torch.equal(a, b)
    q = dev(rng.standard_normal((sum(lens), 8, 64)), torch.float32)
    start = np.concatenate([[0], np.cumsum(lens)])
    r, keep = c.rows(start, first, sum(lens))
    for a, b in zip(every_call(c, r, q, "f32"), every_call(big, r, q, "f32")):
        assert torch.equal(a, b)


@pytest.mark.parametrize("lens", [[1, 1, 1, 1], [3, 2, 1, 4], [30, 20, 9, 25]])
def test_a_table_row_of_several_sequences(lens):
    """The same stream read at several places in one call, the same place twice among them."""
    c, rng = filled([900, 400], 2, 17)
    first, which = [870, 120, 120, 300], [0, 0, 0, 1]
    start = np.concatenate([[0], np.cumsum(lens)])
    q = dev(rng.standard_normal((sum(lens), 8, 64)), torch.float32)
    q[start[2]:start[2] + 1] = q[start[1]:start[1] + 1]
    r, keep = c.rows(start, first, sum(lens), which)
    out, blocks, listed = every_call(c, r, q, "f32")
    assert torch.equal(blocks[start[1]], blocks[start[2]]) and torch.equal(listed[start[1]], listed[start[2]])
    if lens[1] == lens[2]:  # (how the keys are cut up depends on a sequence's last row)
        assert torch.equal(out[start[1]], out[start[2]])
    qf, lists = q.double().cpu().numpy(), blocks.cpu().numpy()
    for s in range(4):
        at = slice(start[s], start[s + 1])
        k, v = c.ref.values(which[s], first[s] + lens[s])
        e, half = bound(qf[at], k, v, 0.125, "f32")
        for got, want in ((out[at], kv4.attend(qf[at], k, v, 0.125, first[s])),
                          (listed[at], listed_reference(qf[at], k, v, 0.125, first[s], lists[at], 2))):
            assert (np.abs(got.double().cpu().numpy() - want) <= e + half * (np.abs(want) + e)).all(), s
        for i in range(lens[s]):
            for h in range(2):
                want = kv8.select(qf[start[s] + i, 4 * h:4 * h + 4], [p[h] for p in c.ref.blocks[which[s]]], first[s] + i, 6, 1, 2)
                assert np.array_equal(lists[start[s] + i, h], want)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("lens,first", [([1, 1], [300, 77]), ([40, 3], [200, 16])])
def test_columns_of_a_wider_matrix(t, lens, first):
    """Queries, keys and values as one product leaves them, and each by itself."""
    hkv, hq, n = 2, 8, sum(lens)
    wide = torch.randn(n, hq + 2 * hkv, 64, device="cuda:0").to(TYPES[t][1])
    parts = wide[:, :hq], wide[:, hq:hq + hkv], wide[:, hq + hkv:]
    start, results = np.concatenate([[0], np.cumsum(lens)]), []
    for q, k, v in (parts, [x.contiguous() for x in parts]):
        c, rng = filled(first, hkv, 4, max_pages=32)
        c.append(lens, first, k, v, t, ref=False)
        r, keep = c.rows(start, first, n)
        results.append((c.pool, *every_call(c, r, q, t)))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    """With outputs and workspaces of their own, on one pool."""
    c, rng = filled([5000, 3000], 4, 23)
    r, keep = c.rows(None, [4999, 2999], 2)
    qs = [torch.randn(2, 16, 64, device="cuda:0") for _ in "ab"]
    want = [every_call(c, r, q, "f32", 40) for q in qs]
    need = hh.hh_kv8_attention_workspace(c.desc, r, 16)
    sel = hh.hh_kv8_select_workspace(c.desc, r, 16, 40)
    lst = hh.hh_kv8_attention_blocks_workspace(c.desc, r, 16, 40)
    sides = [torch.cuda.Stream() for _ in qs]
    ws = [[torch.full((max(b, 1),), 255, dtype=torch.uint8, device="cuda:0") for b in (need, sel, lst)] for _ in qs]
    out = [[torch.zeros_like(q), torch.zeros(2, 4, 40, dtype=torch.int32, device="cuda:0"), torch.zeros_like(q)] for q in qs]
    torch.cuda.synchronize()
    for turn in range(10):
        for q, s, w, o in zip(qs, sides, ws, out):
            on = s.cuda_stream
            hh.hh_kv8_attention(c.desc, r, q.data_ptr(), hh.HH_F32, 1024, 16, 0.125, None, 0, o[0].data_ptr(), hh.HH_F32, 1024,
                                w[0].data_ptr(), need, on)
            hh.hh_kv8_select(c.desc, r, q.data_ptr(), hh.HH_F32, 1024, 16, None, 0, 40, 1, 2, o[1].data_ptr(), w[1].data_ptr(),
                             sel, on)
            hh.hh_kv8_attention_blocks(c.desc, r, o[1].data_ptr(), 40, q.data_ptr(), hh.HH_F32, 1024, 16, 0.125, None, 0,
                                       o[2].data_ptr(), hh.HH_F32, 1024, w[2].data_ptr(), lst, on)
    torch.cuda.synchronize()
    for a, b in zip(want, out):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
