"""The 8-bit paged cache without a GPU: the oracle's format against its
definition, and every argument that the calls refuse before they touch a device."""
import ctypes

import numpy as np
import pytest

from oracle import kv8
from paper_2606_12154_amd import hh


def test_oracle_values_are_within_half_a_step():
    rng = np.random.default_rng(0)
    for size in (1e-5, 0.3, 1.0, 40.0, 6e4):
        k, v = (rng.uniform(-size, size, (16, 64)) for _ in "kv")
        b = kv8.Block()
        b.put(0, k, v)
        for x, got, e, c in zip((k, v), b.values(), b.exp, b.codes):
            assert np.abs(c).max() <= 127 and np.abs(got - x).max() <= 2.0 ** (e - 1)
            if e > kv8.LOW:
                assert np.abs(x).max() > 127 * 2.0 ** (e - 1), "the least exponent"


def test_oracle_exponents_at_their_borders():
    assert [kv8.exponent(x) for x in (0, 127 * 2.0 ** -20, 127.0, np.nextafter(127.0, 128), 254.0, 1e9)] == [-20, -20, 0, 1, 1, 9]


def test_oracle_rows_that_come_one_by_one():
    """Scales of a page grow and never shrink; a value that was held through
    several steps of its page is off by less than one step of the last."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((16, 64)) * np.exp2(rng.uniform(-6, 3, (16, 1)))
    b, last = kv8.Block(), kv8.LOW
    for i in range(16):
        b.put(i, x[i:i + 1], x[i:i + 1])
        assert b.exp[0] >= (last if i else kv8.LOW) and (b.codes[0][i + 1:] == 0).all()
        last = b.exp[0]
        assert np.abs(b.values()[0][:i + 1] - x[:i + 1]).max() < 2.0 ** b.exp[0]
    assert last == kv8.exponent(np.abs(x).max())
    # Cut back and appended to: what lay behind is gone, the scale stays.
    b.put(3, x[:1] * 1e-3, x[:1] * 1e-3)
    assert b.exp[0] == last and (b.codes[0][4:] == 0).all()
    b.put(0, x[:1] * 1e-3, x[:1] * 1e-3)
    assert b.exp[0] < last


def test_oracle_rows_that_are_not_finite():
    x = np.ones((4, 64))
    x[1, 5], x[2, 6] = np.inf, np.nan
    b = kv8.Block()
    b.put(0, x, np.ones((4, 64)))
    assert b.exp == [-6, -6] and b.bad[0].tolist()[:4] == [False, True, True, False] and not b.bad[1].any()
    assert np.isnan(b.values()[0][1:3]).all() and (b.values()[0][[0, 3]] == 1).all()
    b.put(2, np.ones((1, 64)), np.ones((1, 64)))
    assert b.bad[0].tolist()[:4] == [False, True, False, False]


def test_oracle_block_layout_of_named_codes():
    """The places that the header names, read by hand."""
    k, v = np.zeros((16, 64)), np.zeros((16, 64))
    k[3, 32 + 8 * 2 + 5], k[0, 0] = -1.0, 127.0   # h = 1, g = 2, j = 5
    v[4 * 2 + 1, 4 * 9 + 3] = 2.0                 # g = 2, i = 1, r = 9, j = 3
    b = kv8.Block()
    b.put(0, k, v)
    raw = b.bytes()
    assert raw[0] == 255 and raw[256 * 2 + 16 * 3 + 8 + 5] == 127 and (raw[:1024] != 128).sum() == 2
    assert raw[1024 + 256 * 2 + 16 * 9 + 4 * 3 + 1] == 128 + 64 and (raw[1024:2048] != 128).sum() == 1
    assert raw[2048] == 127 and raw[2048 + 53] == 255
    assert raw[2112:].view(np.float16)[[0, 1, 4]].tolist() == [1.0, 2.0 ** -5, 2.0 ** -4]


def test_oracle_summary_is_the_mean_key():
    rng = np.random.default_rng(2)
    for shift in (0.0, 0.5, 2.0):
        b = kv8.Block()
        b.put(0, rng.standard_normal((16, 64)) + shift * rng.standard_normal(64), np.zeros((16, 64)))
        m, s = b.summary()
        assert np.abs(m).max() <= 127 and np.abs(m * s - b.values()[0].mean(0)).max() <= s / 2
    # Sums at the borders of j.
    for top, j in ((127, 0), (128, 1), (254, 1), (255, 2), (508, 2), (509, 3), (1016, 3), (1017, 4), (2032, 4)):
        b = kv8.Block()
        b.exp[0] = 0
        b.codes[0][:, 7] = [top // 16 + (i < top % 16) for i in range(16)]
        m, s = b.summary()
        assert s == 2.0 ** (j - 4) and m[7] == np.rint(top / 2.0 ** j)


def test_oracle_selection():
    rng = np.random.default_rng(3)
    cache = kv8.Cache(1, 12, 1)
    x = rng.standard_normal((12 * 16, 1, 64)) + np.repeat(rng.standard_normal((12, 1, 64)), 16, 0)
    cache.append(0, 0, x, x)
    blocks = [p[0] for p in cache.blocks[0]]
    q = rng.standard_normal((3, 64))
    assert kv8.select(q, blocks, 16 * 4 + 3, 6, 1, 2).tolist() == [0, 1, 2, 3, 4, -1]
    assert kv8.select(q, blocks, -1, 2, 0, 1).tolist() == [-1, -1]
    got = kv8.select(q, blocks, 12 * 16 - 1, 5, 1, 2)
    assert got[0] == 0 and got[3:].tolist() == [10, 11] and sorted(set(got)) == got.tolist()
    mean = np.array([b.values()[0].mean(0) @ q.sum(0) for b in blocks[1:10]])
    assert set(got[1:3] - 1) == set(np.argsort(-mean)[:2]), "the mean keys' order (its gaps are wide here)"
    # Equal scores: the lowest blocks.
    assert kv8.select(q * 0, blocks, 191, 5, 0, 1).tolist() == [0, 1, 2, 3, 11]
    assert kv8.select(q * np.nan, blocks, 191, 3, 0, 1).tolist() == [0, 1, 11]


def test_oracle_query_codes():
    q = np.zeros((2, 64))
    q[0, :4] = [100.0, 0.5, 1.5, -2.5]
    q[1, 0] = 27.0
    assert kv8.query_codes(q)[:4].tolist() == [127, 0, 2, -2]
    q[1, 0] = 27.0 + 1e-9
    assert kv8.query_codes(q)[:4].tolist() == [64, 0, 1, -1]
    assert np.array_equal(kv8.query_codes(q * 2.0 ** -90), kv8.query_codes(q))


# ------------------------------------------------------------------ refusals

A = 1 << 20  # an aligned address that no call here may read


def pool(**kw):
    f = dict(pool=A, page_table=A, n_pages=9, n_kv_heads=2, max_pages=4, table_rows=3)
    f.update(kw)
    return hh.hh_kv8_pool(**f)


def rows(**kw):
    f = dict(row_start=None, first_pos=A, table_row=None, n_seqs=3, n_rows=3, max_rows=1)
    f.update(kw)
    return hh.hh_kv8_rows(**f)


def refused(f, *args, status=hh.HH_ERR_INVALID_ARG):
    with pytest.raises(hh.HHError) as e:
        f(*args)
    assert e.value.status == status


def attention(p, r, q=A, t=2, qs=256, h=4, scale=1.0, rope=None, n=0, o=A, ot=2, os=256, ws=A, size=1 << 30, **status):
    refused(hh.hh_kv8_attention, p, r, q, t, qs, h, scale, rope, n, o, ot, os, ws, size, None, **status)


def listed(p, r, b=A, nb=4, q=A, t=2, qs=256, h=4, scale=1.0, rope=None, n=0, o=A, ot=2, os=256, ws=A, size=1 << 30, **status):
    refused(hh.hh_kv8_attention_blocks, p, r, b, nb, q, t, qs, h, scale, rope, n, o, ot, os, ws, size, None, **status)


def selection(p, r, q=A, t=2, qs=256, h=4, rope=None, n=0, nb=4, first=1, last=1, o=A, ws=A, size=1 << 30, **status):
    refused(hh.hh_kv8_select, p, r, q, t, qs, h, rope, n, nb, first, last, o, ws, size, None, **status)


BAD_POOL = [dict(pool=0), dict(pool=A + 8), dict(page_table=0), dict(page_table=A + 2), dict(n_pages=0),
            dict(n_kv_heads=0), dict(n_kv_heads=-1), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(table_rows=0)]
BAD_ROWS = [dict(first_pos=0), dict(first_pos=A + 1), dict(row_start=A + 2), dict(table_row=A + 1), dict(n_seqs=0),
            dict(n_rows=0), dict(n_rows=2), dict(n_rows=1 << 30), dict(max_rows=0), dict(max_rows=1 << 30)]


@pytest.mark.parametrize("p,r", [(x, {}) for x in BAD_POOL] + [({}, x) for x in BAD_ROWS])
def test_bad_descriptions(p, r):
    p, r = pool(**p), rows(**r)
    refused(hh.hh_kv8_append, p, r, A, A, hh.HH_F16, 128, 128, None, 0, None)
    refused(hh.hh_kv8_read, p, r, A, A, hh.HH_F16, 128, 128, None)
    attention(p, r)
    listed(p, r)
    selection(p, r)


@pytest.mark.parametrize("k,v,t,ks,vs", [
    (0, A, 2, 128, 128), (A, 0, 2, 128, 128), (A + 8, A, 2, 128, 128), (A, A + 4, 2, 128, 128), (A, A, 3, 128, 128),
    (A, A, -1, 128, 128), (A, A, 2, 127, 128), (A, A, 2, 128, 132), (A, A, 0, 130, 128), (A, A, 1, 120, 128),
    (A, A, 2, -128, 128)])
def test_append_and_read_refuse(k, v, t, ks, vs):
    refused(hh.hh_kv8_append, pool(), rows(), k, v, t, ks, vs, None, 0, None)
    refused(hh.hh_kv8_read, pool(), rows(), k, v, t, ks, vs, None)


def test_rope_tables_refused():
    for at, n in ((A + 4, 9), (A, 0), (A, -1)):
        refused(hh.hh_kv8_append, pool(), rows(), A, A, 2, 128, 128, at, n, None)
        for call in (attention, listed, selection):
            call(pool(), rows(), rope=at, n=n)


@pytest.mark.parametrize("bad", [
    dict(q=0), dict(o=0), dict(o=A + 8), dict(t=4), dict(ot=-1), dict(h=3), dict(h=0), dict(h=-2), dict(qs=255), dict(os=192),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=2.0 ** 101)])
def test_attention_refuses(bad):
    attention(pool(), rows(), **bad)
    listed(pool(), rows(), **bad)


def test_listed_blocks_refused():
    for bad in (dict(b=0), dict(b=A + 2), dict(nb=0), dict(nb=-1)):
        listed(pool(), rows(), **bad)
    listed(pool(), rows(), nb=(1 << 15) + 1, status=hh.HH_ERR_UNSUPPORTED)


@pytest.mark.parametrize("bad", [
    dict(q=0), dict(q=A + 8), dict(t=3), dict(h=3), dict(h=0), dict(qs=255), dict(o=0), dict(o=A + 1), dict(nb=0), dict(nb=-4),
    dict(first=-1), dict(last=0), dict(last=-1), dict(first=4), dict(first=2, last=3), dict(first=(1 << 31) - 1, last=(1 << 31) - 1)])
def test_selection_refuses(bad):
    selection(pool(), rows(), **bad)


def test_selections_too_large():
    selection(pool(), rows(), nb=(1 << 15) + 1, status=hh.HH_ERR_UNSUPPORTED)
    selection(pool(max_pages=(1 << 15) + 1), rows(), status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv8_select_workspace, pool(max_pages=(1 << 15) + 1), rows(), 4, 4, status=hh.HH_ERR_UNSUPPORTED)
    big = rows(row_start=A, n_seqs=1 << 20, n_rows=1 << 29, max_rows=1 << 29)
    selection(pool(), big, status=hh.HH_ERR_UNSUPPORTED)


@pytest.mark.parametrize("ask,call", [
    (lambda p, r: hh.hh_kv8_attention_workspace(p, r, 4), attention),
    (lambda p, r: hh.hh_kv8_select_workspace(p, r, 4, 400), lambda p, r, **kw: selection(p, r, nb=400, **kw)),
    (lambda p, r: hh.hh_kv8_attention_blocks_workspace(p, r, 4, 400), lambda p, r, **kw: listed(p, r, nb=400, **kw))])
def test_workspaces(ask, call):
    p, r = pool(n_pages=30000, max_pages=9000), rows()
    need = ask(p, r)
    assert 0 < need <= hh.HH_KV8_WORKSPACE_MOST
    for at, n in ((A, need - 1), (None, need), (A + 64, need)):
        call(p, r, ws=at, size=n)
    refused(ask, pool(n_kv_heads=3), r)
    refused(ask, pool(n_kv_heads=0), r)


def test_workspace_queries_without_places():
    lib = hh.load_library()
    p, r = pool(), rows()
    for f, more in ((lib.hh_kv8_attention_workspace, ()), (lib.hh_kv8_select_workspace, (4,)), (lib.hh_kv8_attention_blocks_workspace, (4,))):
        n = ctypes.c_size_t()
        assert f(ctypes.byref(p), ctypes.byref(r), 4, *more, ctypes.byref(n)) == hh.HH_OK
        for a, b, c in ((None, ctypes.byref(r), ctypes.byref(n)), (ctypes.byref(p), None, ctypes.byref(n)), (ctypes.byref(p), ctypes.byref(r), None)):
            assert f(a, b, 4, *more, c) == hh.HH_ERR_INVALID_ARG
        if more:
            assert f(ctypes.byref(p), ctypes.byref(r), 4, 0, ctypes.byref(n)) == hh.HH_ERR_INVALID_ARG


def test_calls_too_large_for_a_launch():
    big = rows(row_start=A, n_seqs=1 << 20, n_rows=1 << 29, max_rows=1 << 29)
    refused(hh.hh_kv8_append, pool(), big, A, A, 2, 128, 128, None, 0, None, status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv8_read, pool(), big, A, A, 2, 128, 128, None, status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv8_attention_workspace, pool(), big, 4, status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv8_attention_blocks_workspace, pool(), big, 4, 4, status=hh.HH_ERR_UNSUPPORTED)
    wide = pool(n_kv_heads=1)
    attention(wide, rows(n_seqs=1, n_rows=1), h=1 << 25, qs=1 << 31, os=1 << 31, status=hh.HH_ERR_UNSUPPORTED)
    listed(wide, rows(n_seqs=1, n_rows=1), h=1 << 25, qs=1 << 31, os=1 << 31, status=hh.HH_ERR_UNSUPPORTED)


# ------------------------------------------------------------------ contexts with an 8-bit cache

def test_cache_format_in_the_config():
    import synth
    for f in (0, hh.HH_WF_Q4G32):
        n, c, sh = 4, 4096, synth.ONE_B
        sizes = [hh.hh_workspace_size(hh.make_config(sh, n, c, 512, weight_format=f + k)) for k in (0, hh.HH_KV_Q4, hh.HH_KV_Q8)]
        kv = n * c * sh.n_layers * sh.n_kv_heads
        assert abs(sizes[2] - sizes[1] - kv * (136 - 72)) < 4096
        extra = 512 * (sh.q_dim + 2 * sh.kv_dim) * 4 + (16 << 20)  # the pass's fp32 rows and split outputs
        assert abs(sizes[0] - sizes[2] - (kv * (256 - 136) - extra)) < 4096
    for bad in (hh.HH_KV_Q8 + hh.HH_KV_Q4, hh.HH_KV_Q8 + 2, hh.HH_KV_Q8 + hh.HH_WF_Q4G32, hh.HH_KV_Q8 + 0x200):
        with pytest.raises(hh.HHError) as e:
            hh.hh_workspace_size(hh.make_config(synth.TINY, 2, 128, weight_format=bad))
        assert e.value.status == hh.HH_ERR_UNSUPPORTED
    assert hh.hh_workspace_size(hh.make_config(synth.TINY, 2, 128, weight_format=hh.HH_KV_Q8)) > 0
