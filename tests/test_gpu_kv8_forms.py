"""Attention over the 8-bit paged cache by every kernel and way of cutting a call up (test_kv8_cases.py
holds the cases to that).

* Element by element against fp64 attention over the values that the pages hold, within the bound
  of test_gpu_kv4_forms.py, whose kernels these share weights and sums with.  Queries of few columns are
  whole numbers of 23 bits: 2^-22 of the largest |q| for each element, 2^-22 x 5 of sum |q_i k_i| in rows of 64
  N(0, 1) elements (the largest is below 4, the mean 0.8), and their products are exact, so that the
  2^-18 that the bound holds for sums of products covers them.
* Counts: with queries of 0 all weights are one number, 2^12, and sums of them exact below 2^24; values are 1 in
  one dimension, by the block or by the slot, and 0 elsewhere. The result is the share of the attended positions
  that have that dimension, but for a reciprocal and a product, 2^-24 each, and half a step of the type. A position
  that is left out, or taken twice, moves it by 2^-15 and more.
"""
import numpy as np
import pytest

from kv4_cases import CASES
from kv8_cases import LISTS, LONG
from paper_2606_12154_amd import hh
from test_gpu_kv4_forms import HALF_STEP, check
from test_gpu_kv8 import TYPES, Cache, attend, bound, dev, ints, listed_reference, read, rope_table, select, stream

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def some_rows(n, sample):
    """The first and last rows, and others between them."""
    which = torch.arange(n)
    if n <= sample:
        return which
    return torch.cat([which[:sample // 2], torch.randperm(n - 1)[:sample - sample // 2 - 1], which[-1:]]).unique()


def fill(lens, hkv, seed, max_pages, k=None, v=None):
    c = Cache(len(lens), hkv, max_pages or (max(max(lens), 1) + 15) // 16, seed)
    n = sum(lens)
    k = torch.randn(n, hkv, 64, device="cuda:0") if k is None else k
    v = torch.randn(n, hkv, 64, device="cuda:0") if v is None else v
    c.append(lens, [0] * len(lens), k, v, "f32", ref=False)
    return c


def run(rows, first, hkv, group, t, ot, rope, seed, max_pages=None, sample=40, marked=(), shared=False):
    """rows[i] rows of sequence i from position first[i] on (which may be negative); marked: (sequence,
    position) of keys that are not finite; shared: all of one stream."""
    torch.manual_seed(seed)
    lens, hq = [max(r + f, 0) for r, f in zip(rows, first)], hkv * group
    if shared:
        lens = [max(lens)]
    at, start = np.concatenate([[0], np.cumsum(lens)]), np.concatenate([[0], np.cumsum(rows)])
    k = torch.randn(sum(lens), hkv, 64, device="cuda:0")
    for s, p in marked:
        k[at[s] + p, :, 3] = float("inf")
    c = fill(lens, hkv, seed, max_pages, k=k)
    kk, vv = (a.double() for a in read(c, lens, [0] * len(lens), "f32"))
    n = int(start[-1])
    q = torch.randn(n, hq, 64, device="cuda:0").to(TYPES[t][1])
    out = torch.full(q.shape, 3.0, dtype=TYPES[ot][1], device="cuda:0")
    tab = rope_table(max(max(lens), 1)) if rope else None
    r, keep = c.rows(start, first, n, [0] * len(rows) if shared else None)
    attend(c, r, q, t, out, ot, 0.125, tab)
    at = [0] * len(rows) if shared else at
    for i in some_rows(len(rows), 8).tolist() if shared else range(len(rows)):
        which = some_rows(rows[i], sample)
        pos = which + first[i]
        got = out[(which + int(start[i])).cuda()].double()
        assert (got[(pos < 0).cuda()] == 0).all()
        bad = torch.zeros(len(which), dtype=torch.bool)
        for s, p in marked:
            bad |= (s == i) & (pos >= p)
        assert torch.isnan(got[bad.cuda()]).all()
        ok = ~bad & (pos >= 0)
        if not ok.any():
            continue
        top = int(pos[ok].max()) + 1
        check(got[ok.cuda()], q[(which[ok] + int(start[i])).cuda()].double(), kk[at[i]:at[i] + top], vv[at[i]:at[i] + top], 0.125,
              pos[ok].cuda(), ot, None if tab is None else dev(tab))


TYPE_PAIRS = [("f16", "f16", False), ("bf16", "bf16", False), ("f32", "f32", False), ("f32", "bf16", False), ("bf16", "f32", True),
              ("f32", "f16", True)]


@pytest.mark.parametrize("t,ot,rope", TYPE_PAIRS)
@pytest.mark.parametrize("case", list(CASES))
def test_every_kernel(case, t, ot, rope):
    """Queries of one term, of two and of whole numbers through every kernel and way of cutting a call up."""
    rows, first, hkv, group, pages = CASES[case]
    run(rows, first, hkv, group, t, ot, rope, seed=7, max_pages=pages)


@pytest.mark.parametrize("t,ot,rope", [("f16", "f32", False), ("f32", "f32", False), ("bf16", "f32", True)])
@pytest.mark.parametrize("rows,first,hkv,group", [([1400, 9, 700, 3], [-5, -4, 0, -3], 4, 4), ([40] * 24, [i % 9 - 4 for i in range(24)], 8, 4),
                                                  ([33, 33], [-40, -1], 8, 4), ([300, 1, 0, 77], [0, -1, 3, -76], 8, 4)])
def test_prompts_with_padding(t, ot, rope, rows, first, hkv, group):
    """Tiles of one, two and four columns whose rows are at negative positions, in part or all."""
    run(rows, first, hkv, group, t, ot, rope, seed=3)


@pytest.mark.parametrize("t,rope", [("f16", False), ("f32", False), ("bf16", True)])
@pytest.mark.parametrize("rows,first", [([1999], [0]), ([300], [40]), ([64, 40], [3005, 0]), ([12], [50])])
def test_marked_slots_in_tiles(t, rope, rows, first):
    """A key that is not finite, seen by the last rows of a tile alone, or by all of them."""
    n = rows[0] + first[0]
    for p in (n - 1, n - 1 - rows[0] // 2, first[0]):
        run(rows, first, 8, 4, t, "f32", rope, seed=p, marked=[(0, p)])


# ------------------------------------------------------------------ counts

def count(rows, first, hkv, group, t, ot, pages=None, lists=None, shared=False):
    """Every attended position counts once (or as often as it is listed)."""
    lens, start = [r + f for r, f in zip(rows, first)], np.concatenate([[0], np.cumsum(rows)])
    n, hq = int(start[-1]), hkv * group
    held = [max(lens)] if shared else lens
    pos = torch.cat([torch.arange(m) for m in held]).cuda()
    k = torch.randn(len(pos), hkv, 64, device="cuda:0")
    q = torch.zeros(n, hq, 64, device="cuda:0").to(TYPES[t][1])
    for of in (pos // 16 % 64, (pos + pos // 16) % 64):
        v = torch.nn.functional.one_hot(of, 64).float()[:, None].repeat(1, hkv, 1)
        c = fill(held, hkv, 1, pages, k=k, v=v)
        out = torch.full(q.shape, 3.0, dtype=TYPES[ot][1], device="cuda:0")
        r, keep = c.rows(start, first, n, [0] * len(rows) if shared else None)
        attend(c, r, q, t, out, ot, blocks=None if lists is None else ints(lists))
        got, at = out.double(), 0
        for i in range(len(rows)):
            one = v[at:at + lens[i], 0].double()
            at += 0 if shared else lens[i]
            p = torch.arange(rows[i]).cuda() + first[i]
            if lists is None:
                want = one.cumsum(0)[p][:, None].expand(-1, hkv, -1)
            else:
                # How often each position is listed, and seen.
                some = dev(lists[start[i]:start[i + 1]].astype(np.int64))
                nb = (lens[i] + 15) // 16
                times = torch.zeros(rows[i], hkv, nb + 1, device="cuda:0", dtype=torch.float64)
                inside = (some >= 0) & (some <= (p // 16)[:, None, None])
                times.scatter_add_(2, torch.where(inside, some, nb), torch.ones_like(some, dtype=torch.float64))
                times = times[..., :nb].repeat_interleave(16, -1)[..., :lens[i]]
                times *= (torch.arange(lens[i]).cuda() <= p[:, None])[:, None]
                want = times @ one
            total = want.sum(-1, keepdim=True)
            want = torch.where(total > 0, want / total.clamp(min=1), torch.zeros((), device="cuda:0", dtype=torch.float64))
            want = want.repeat_interleave(group, 1)
            tol = want * (2.0 ** -22 + HALF_STEP[ot] * (1 + 2.0 ** -22)) + 2.0 ** -25 * (ot == "f16")
            err = (got[start[i]:start[i + 1]] - want).abs()
            assert (err <= tol).all(), (i, (err - tol).max().item(), want.max().item())


@pytest.mark.parametrize("t,ot", [("f16", "f32"), ("f32", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("case", list(CASES))
def test_counts_by_every_kernel(case, t, ot):
    rows, first, hkv, group, pages = CASES[case]
    count(rows, first, hkv, group, t, ot, pages)


@pytest.mark.parametrize("t", ["f16", "f32"])
@pytest.mark.parametrize("case", list(LONG))
def test_counts_over_many_steps(case, t):
    """Waves that take more than 64 steps, whose page ids are read anew."""
    rows, first, hkv, group, pages = LONG[case]
    count(rows, first, hkv, group, t, "f32", pages, shared=True)


@pytest.mark.parametrize("t,ot,rope", [("f16", "f16", False), ("f32", "f32", False), ("bf16", "f32", True)])
@pytest.mark.parametrize("case", list(LONG))
def test_values_over_many_steps(case, t, ot, rope):
    rows, first, hkv, group, pages = LONG[case]
    run(rows, first, hkv, group, t, ot, rope, seed=2, max_pages=pages, sample=4, shared=True)


def random_lists(rows, first, hkv, n, kind, rng):
    """Blocks of each row and head in any order, with entries that are none; "late": the row's own block and
    most others behind the first 128 entries, "twice": the same ones again."""
    out = np.full((rows, hkv, n), -1, np.int32)
    for i in range(rows):
        p = first + i
        for h in range(hkv):
            some = rng.permutation(p // 16)[:n - 1]
            keep = rng.random(len(some)) < (0.03 if kind == "late" else 0.8)
            if kind == "late" and len(some) > 140:
                keep[128:] = rng.random(len(some) - 128) < 0.9
            some = np.where(keep, some, rng.choice([-1, -9, p // 16 + 1, 1 << 30]))
            out[i, h, :len(some)] = some
            out[i, h, len(some) if kind == "late" else 0] = p // 16
            if kind == "twice":
                out[i, h, -(n // 3):] = out[i, h, :n // 3]
    return out


@pytest.mark.parametrize("t", ["f16", "f32"])
@pytest.mark.parametrize("kind", ["some", "late", "twice"])
@pytest.mark.parametrize("case", list(LISTS))
def test_counts_of_listed_blocks(case, kind, t):
    """Lists by every way of cutting them up, and over more steps than a wave holds at once."""
    rows, first, hkv, group, n = LISTS[case]
    count([rows], [first], hkv, group, t, "f32", lists=random_lists(rows, first, hkv, n, kind, np.random.default_rng(rows + n)))


@pytest.mark.parametrize("t,rope", [("f16", False), ("f32", False), ("bf16", True)])
@pytest.mark.parametrize("case", list(LISTS))
def test_values_of_listed_blocks(case, t, rope):
    """Rows and heads one by one, against the attention over the positions that are listed, within the bound of the
    attention over all keys at that number of keys."""
    rows, first, hkv, group, n = LISTS[case]
    torch.manual_seed(5)
    lists = random_lists(rows, first, hkv, n, "late" if n > 128 else "some", np.random.default_rng(n))
    c = fill([first + rows], hkv, 5, None)
    kk, vv = (a.double() for a in read(c, [first + rows], [0], "f32"))
    tab = rope_table(first + rows) if rope else None
    q = torch.randn(rows, hkv * group, 64, device="cuda:0").to(TYPES[t][1])
    out = torch.full(q.shape, 3.0, device="cuda:0")
    r, keep = c.rows([0, rows], [first], rows)
    attend(c, r, q, t, out, "f32", rope=tab, blocks=ints(lists))
    for i in some_rows(rows, 6).tolist():
        p, rot = first + i, q[i:i + 1].double()
        length = None
        if tab is not None:
            co, si = dev(tab)[p].double().unbind(-1)
            x, y = rot[..., :32], rot[..., 32:]
            length = torch.sqrt(x * x + y * y).repeat(1, 1, 2)
            rot = torch.cat([x * co - y * si, y * co + x * si], -1)
        for h in range(hkv):
            blocks = np.array([b for b in lists[i, h] if 0 <= b <= p // 16])
            at = (blocks[:, None] * 16 + np.arange(16)).ravel()
            at = dev(at[at <= p])
            heads = slice(h * group, (h + 1) * group)
            mine = rot[:, heads]
            kh, vh = kk[at, h], vv[at, h]
            w = torch.softmax(mine[0] @ kh.T.contiguous() * 0.125, -1)
            ref, s = w @ vh, w @ vh.abs()
            a = ((mine if length is None else length[:, heads])[0].abs() @ kh.abs().T.contiguous() * 0.125).amax(-1, keepdim=True)
            e = 2.0 ** -17.5 * a + 2.0 ** -18.5
            m = len(at)
            e = (2 * e + 2 * (m / 32 + n / 2 + 16) * 2.0 ** -24) * s + 2.0 ** -36 * m * vh.abs().max()
            err = (out[i, heads].double() - ref).abs() - (e + HALF_STEP["f32"] * (ref.abs() + e))
            assert (err <= 0).all(), (i, h, err.max().item())


# ------------------------------------------------------------------ captured selections

@pytest.mark.parametrize("pages,rows,n", [(3000, [1, 1, 1], 40), (9000, [1, 1], 100), (30000, [1], 64), (2000, [9, 30], 20), (17000, [1] * 40, 30)])
def test_captured_selections_replay(pages, rows, n):
    """Scores in a launch of their own, and scores that take more LDS than a kernel has unasked: every replay equals
    the eager call on what the inputs hold then, with eager calls and other widths between."""
    hkv, hq, m = 2, 8, sum(rows)
    c = Cache(1, hkv, pages, 0, spare=0)
    c.d_table = ints(np.tile(np.arange(pages), (len(rows), 1)))  # (one stream's pages, read at several places)
    c.desc = hh.hh_kv8_pool(c.pool.data_ptr(), c.d_table.data_ptr(), c.n_pages, hkv, pages, len(rows))
    x = [torch.randn(pages * 16, hkv, 64, device="cuda:0") for _ in "kv"]
    r, keep = c.rows([0, pages * 16], [0], pages * 16)
    hh.hh_kv8_append(c.desc, r, x[0].data_ptr(), x[1].data_ptr(), hh.HH_F32, 128, 128, None, 0, stream())
    first = ints([pages * 16 - k - 17 * i - 40 for i, k in enumerate(rows)])
    start = ints(np.concatenate([[0], np.cumsum(rows)]))
    r = hh.hh_kv8_rows(start.data_ptr(), first.data_ptr(), None, len(rows), m, max(rows))
    small = hh.hh_kv8_pool(c.pool.data_ptr(), c.d_table.data_ptr(), c.n_pages, hkv, 2100, 1)
    one = hh.hh_kv8_rows(None, ints([2100 * 16 - 1]).data_ptr(), None, 1, 1, 1) if pages > 2100 else None
    q, out = torch.zeros(m, hq, 64, device="cuda:0"), torch.zeros(m, hkv, n, dtype=torch.int32, device="cuda:0")
    need = hh.hh_kv8_select_workspace(c.desc, r, hq, n)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda:0")
    call = lambda: hh.hh_kv8_select(c.desc, r, q.data_ptr(), hh.HH_F32, hq * 64, hq, None, 0, n, 1, 2, out.data_ptr(), ws.data_ptr(), need, stream())
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for turn in range(5):
        q.normal_()
        first += 3
        out.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        if one is not None:
            c2 = type("C", (), dict(desc=small, hkv=hkv))
            one_first = ints([2100 * 16 - 1 - turn])
            one = hh.hh_kv8_rows(None, one_first.data_ptr(), None, 1, 1, 1)
            select(c2, one, torch.randn(1, hq, 64, device="cuda:0"), "f32", n, 1, 2)
        out.fill_(-7)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and (got >= 0).all() and (got[..., 1:] > got[..., :-1]).all()


# ------------------------------------------------------------------ whatever lies in pages that no row sees

@pytest.mark.parametrize("bits", [0xffff, 0xbc00, 0x3c00, 0x7c00, 0xfc00, 0x0000, 0x8000, 0xfbff, 0x7bff])
@pytest.mark.parametrize("group", [4, 12])
def test_entries_that_are_none_beside_any_bytes(bits, group):
    """A sequence whose first pages were never written, and lists of its others with entries that are none:
    the page that is read in their place may have any scale, negative and infinite ones too."""
    torch.manual_seed(1)
    c = Cache(1, 1, 6)
    c.pool.view(torch.int16).fill_(bits - (bits >> 15 << 16))
    k, v = (torch.randn(64, 1, 64, device="cuda:0") for _ in "kv")
    c.append([64], [32], k, v, "f32")
    lists = np.array([[2, -1, -1, 3, 5, -1, -1, -1], [-1, -1, 4, -1, -1, 99, 2, -1], [5, -1, -1, -1, -1, -1, -1, -1]], np.int32)[:, None]
    q = torch.randn(3, group, 64, device="cuda:0")
    out = torch.full(q.shape, 3.0, device="cuda:0")
    r, keep = c.rows([0, 3], [93], 3)
    attend(c, r, q, "f32", out, "f32", blocks=ints(lists))
    want = listed_reference(q.double().cpu().numpy(), *c.ref.values(0, 96), 0.125, 93, lists, 1)
    e, half = bound(q.double().cpu().numpy(), *(x[32:] for x in c.ref.values(0, 96)), 0.125, "f32")
    assert (np.abs(out.double().cpu().numpy() - want) <= e + half * (np.abs(want) + e)).all()
