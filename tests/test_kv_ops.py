"""The 4-bit paged cache and the page operators without a GPU: the oracle's
format against its definition, and every argument that the calls refuse
before they touch a device."""
import ctypes

import numpy as np
import pytest

from oracle import kv4
from paper_2606_12154_amd import hh


def test_oracle_values_are_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((500, 64)) * np.exp(rng.uniform(-9, 7, (500, 1)))).astype(np.float32)
    c, s = kv4.quantize(x)
    v = kv4.dequantize(c, s)
    assert np.abs(c).max() == 7
    # The scale is max / 7 to 2^-8 of itself and the quotient to 2^-24, so a
    # code is within half a step, and the largest within 7 * 2^-8 of one.
    half = np.repeat(s, 32, axis=-1) * (0.5 + 7 * 2.0 ** -8)
    assert (np.abs(v - x) <= half).all()
    assert np.array_equal(v, v.astype(np.float16).astype(np.float64)), "values are fp16 numbers"
    assert np.array_equal(24 * s, (24 * s).astype(np.float16).astype(np.float64)), "24 s is one too"


def test_oracle_special_rows():
    x = np.zeros((6, 64), np.float32)
    x[1, :6] = [7.0, 2.5, 3.5, -2.5, -0.5, 6.5]   # s = 1: ties to even
    x[2, :32] = 1e-9                              # below half of 2^-24 times 7
    x[2, 32:] = 3 * 2.0 ** -22
    x[3, 0], x[3, 40] = 1e6, -3e38
    x[4, 5] = np.inf
    x[5, 63] = np.nan
    c, s = kv4.quantize(x)
    assert c[1, :6].tolist() == [7, 2, 4, -2, 0, 6] and (c[0] == 0).all() and (s[0] == 0).all()
    assert s[2, 0] == 0 and (c[2, :32] == 0).all() and s[2, 1] == 2 * 2.0 ** -24 and (c[2, 32:] == 6).all()
    assert (s[3] == 2720).all() and c[3, 0] == 7 and c[3, 40] == -7
    assert np.isnan(s[4]).all() and np.isnan(s[5]).all()


def test_oracle_block_is_a_permutation():
    """Every code and scale has a place of its own."""
    rng = np.random.default_rng(1)
    k, v = (rng.standard_normal((16, 64)).astype(np.float32) for _ in range(2))
    a, b = np.zeros(kv4.BLOCK, np.uint8), np.full(kv4.BLOCK, 255, np.uint8)
    for i in rng.permutation(16):
        kv4.put(a, i, k[i], v[i])
    for i in rng.permutation(16):
        kv4.put(b, i, k[i], v[i])
    assert np.array_equal(a, b)
    n = np.stack([a[:1024] & 15, a[:1024] >> 4]).astype(int).reshape(2, 2, 512) - 8
    for x, got in ((k, n[:, 0]), (v, n[:, 1])):
        assert np.array_equal(np.sort(kv4.quantize(x)[0].ravel()), np.sort(got.ravel()))


def test_oracle_block_layout_of_named_codes():
    """The places that the header names, read by hand."""
    k, v = np.zeros((1, 64), np.float32), np.zeros((1, 64), np.float32)
    k[0, 0], k[0, 32 + 8 * 2 + 5] = 7, -7   # t = 1, g = 2, j = 2, h = 1
    v[0, 4 * 9 + 3], v[0, 0] = 7, 7
    b = np.full(kv4.BLOCK, 0x88, np.uint8)
    b[1024:] = 0
    kv4.put(b, 6, k[0], v[0])
    w = b[:1024].view(np.uint16)
    assert w[4 * (16 * 0 + 6)] == 0x888f
    assert w[4 * (16 * 2 + 6) + 3] == 0x8188
    assert w[256 + 4 * (16 * 1 + 9) + 2] == 0xf888 and w[256 + 4 * 16 + 2] == 0x888f
    s = b[1024:].view(np.float16)
    assert s[12] == 1 and s[13] == 1 and s[32 + 6] == 1 and s[48 + 6] == 1 and (s != 0).sum() == 4


# ------------------------------------------------------------------ refusals

A = 1 << 20  # an aligned address that no call here may read


def pool(**kw):
    f = dict(pool=A, page_table=A, n_pages=9, n_kv_heads=2, max_pages=4, table_rows=3)
    f.update(kw)
    return hh.hh_kv4_pool(**f)


def rows(**kw):
    f = dict(row_start=None, first_pos=A, table_row=None, n_seqs=3, n_rows=3, max_rows=1)
    f.update(kw)
    return hh.hh_kv4_rows(**f)


def refused(f, *args, status=hh.HH_ERR_INVALID_ARG):
    with pytest.raises(hh.HHError) as e:
        f(*args)
    assert e.value.status == status


BAD_POOL = [dict(pool=0), dict(pool=A + 8), dict(page_table=0), dict(page_table=A + 2), dict(n_pages=0),
            dict(n_kv_heads=0), dict(n_kv_heads=-1), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(table_rows=0)]
BAD_ROWS = [dict(first_pos=0), dict(first_pos=A + 1), dict(row_start=A + 2), dict(table_row=A + 1), dict(n_seqs=0),
            dict(n_rows=0), dict(n_rows=2), dict(n_rows=1 << 30), dict(max_rows=0), dict(max_rows=1 << 30)]


@pytest.mark.parametrize("p,r", [(x, {}) for x in BAD_POOL] + [({}, x) for x in BAD_ROWS])
def test_bad_descriptions(p, r):
    p, r = pool(**p), rows(**r)
    refused(hh.hh_kv4_append, p, r, A, A, hh.HH_F16, 128, 128, None, 0, None)
    refused(hh.hh_kv4_read, p, r, A, A, hh.HH_F16, 128, 128, None)
    refused(hh.hh_kv4_attention, p, r, A, hh.HH_F16, 256, 4, 0.125, None, 0, A, hh.HH_F16, 256, A, 1 << 30, None)


@pytest.mark.parametrize("k,v,t,ks,vs", [
    (0, A, 2, 128, 128), (A, 0, 2, 128, 128), (A + 8, A, 2, 128, 128), (A, A + 4, 2, 128, 128), (A, A, 3, 128, 128),
    (A, A, -1, 128, 128), (A, A, 2, 127, 128), (A, A, 2, 128, 132), (A, A, 0, 130, 128), (A, A, 1, 120, 128),
    (A, A, 2, -128, 128)])
def test_append_and_read_refuse(k, v, t, ks, vs):
    refused(hh.hh_kv4_append, pool(), rows(), k, v, t, ks, vs, None, 0, None)
    refused(hh.hh_kv4_read, pool(), rows(), k, v, t, ks, vs, None)


def test_rope_tables_refused():
    for at, n in ((A + 4, 9), (A, 0), (A, -1)):
        refused(hh.hh_kv4_append, pool(), rows(), A, A, 2, 128, 128, at, n, None)
        refused(hh.hh_kv4_attention, pool(), rows(), A, 2, 256, 4, 0.125, at, n, A, 2, 256, A, 1 << 30, None)


@pytest.mark.parametrize("q,t,qs,h,scale,o,ot,os", [
    (0, 2, 256, 4, 1.0, A, 2, 256), (A, 2, 256, 4, 1.0, 0, 2, 256), (A, 2, 256, 4, 1.0, A + 8, 2, 256),
    (A, 4, 256, 4, 1.0, A, 2, 256), (A, 2, 256, 4, 1.0, A, -1, 256), (A, 2, 256, 3, 1.0, A, 2, 256),
    (A, 2, 256, 0, 1.0, A, 2, 256), (A, 2, 255, 4, 1.0, A, 2, 256), (A, 2, 256, 4, 1.0, A, 2, 192),
    (A, 2, 256, 4, 0.0, A, 2, 256), (A, 2, 256, 4, -1.0, A, 2, 256), (A, 2, 256, 4, float("inf"), A, 2, 256),
    (A, 2, 256, 4, float("nan"), A, 2, 256)])
def test_attention_refuses(q, t, qs, h, scale, o, ot, os):
    refused(hh.hh_kv4_attention, pool(), rows(), q, t, qs, h, scale, None, 0, o, ot, os, A, 1 << 30, None)


def test_attention_workspace():
    p, r = pool(n_pages=1000, max_pages=900), rows()
    need = hh.hh_kv4_attention_workspace(p, r, 4)
    assert need > 0
    for at, n in ((A, need - 1), (None, need), (A + 64, need)):
        refused(hh.hh_kv4_attention, p, r, A, 2, 256, 4, 1.0, None, 0, A, 2, 256, at, n, None)
    assert hh.hh_kv4_attention_workspace(pool(max_pages=1), r, 4) == 0
    refused(hh.hh_kv4_attention_workspace, p, r, 3)
    refused(hh.hh_kv4_attention_workspace, pool(n_kv_heads=0), r, 4)
    lib = hh.load_library()
    assert lib.hh_kv4_attention_workspace(ctypes.byref(p), ctypes.byref(r), 4, None) == hh.HH_ERR_INVALID_ARG
    assert lib.hh_kv4_attention_workspace(None, ctypes.byref(r), 4, None) == hh.HH_ERR_INVALID_ARG
    n = ctypes.c_size_t()
    assert lib.hh_kv4_attention_workspace(ctypes.byref(p), None, 4, ctypes.byref(n)) == hh.HH_ERR_INVALID_ARG


def test_calls_too_large_for_a_launch():
    big = rows(row_start=A, n_seqs=1 << 20, n_rows=1 << 29, max_rows=1 << 29)
    refused(hh.hh_kv4_append, pool(), big, A, A, 2, 128, 128, None, 0, None, status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv4_read, pool(), big, A, A, 2, 128, 128, None, status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv4_attention_workspace, pool(), big, 4, status=hh.HH_ERR_UNSUPPORTED)


@pytest.mark.parametrize("at,layers,stride,size,pages", [
    (0, 1, 0, 1152, 8), (A + 8, 1, 0, 1152, 8), (A, 0, 0, 1152, 8), (A, 1, 0, 1144, 8), (A, 1, 0, 0, 8),
    (A, 1, 0, 1152, 0), (A, 2, 1152 * 8 - 16, 1152, 8), (A, 2, 1152 * 8 + 8, 1152, 8), (A, 1, 0, (1 << 30) + 16, 8)])
def test_page_pools_refused(at, layers, stride, size, pages):
    refused(hh.hh_kv_copy_pages, at, layers, stride, size, pages, [0], [1], None)
    refused(hh.hh_kv_compact, at, layers, stride, size, pages, A, 1, 4, A, A, A, 1 << 30, None)


@pytest.mark.parametrize("src,dst", [([0], [8]), ([8], [0]), ([-1], [0]), ([0], [-1]), ([0, 1], [2, 2]),
                                     ([0, 1], [1, 2]), ([1, 0], [2, 1]), ([3], [3])])
def test_copies_refused(src, dst):
    refused(hh.hh_kv_copy_pages, A, 2, 1152 * 8, 1152, 8, src, dst, None)


def test_copy_of_nothing_and_unequal_lists():
    hh.hh_kv_copy_pages(A, 2, 1152 * 8, 1152, 8, [], [], None)
    with pytest.raises(ValueError):
        hh.hh_kv_copy_pages(A, 2, 1152 * 8, 1152, 8, [0], [1, 2], None)
    lib = hh.load_library()
    assert lib.hh_kv_copy_pages(A, 1, 0, 1152, 8, -1, None, None, None) == hh.HH_ERR_INVALID_ARG
    assert lib.hh_kv_copy_pages(A, 1, 0, 1152, 8, 1, None, None, None) == hh.HH_ERR_INVALID_ARG


def test_compaction_refuses():
    need = hh.hh_kv_compact_workspace(8)
    ok = dict(pool=A, layers=1, stride=0, size=1152, pages=8, table=A, rows=2, cols=4, lens=A, live=A, ws=A, n=need)
    for bad in (dict(table=0), dict(table=A + 2), dict(rows=0), dict(cols=0), dict(lens=0), dict(live=0), dict(live=A + 1),
                dict(ws=0), dict(ws=A + 16), dict(n=need - 1)):
        refused(hh.hh_kv_compact, *{**ok, **bad}.values(), None)
    refused(hh.hh_kv_compact, *{**ok, "pages": (1 << 20) + 1, "n": 1 << 40}.values(), None, status=hh.HH_ERR_UNSUPPORTED)
    refused(hh.hh_kv_compact_workspace, 0)
    refused(hh.hh_kv_compact_workspace, (1 << 20) + 1, status=hh.HH_ERR_UNSUPPORTED)


# ------------------------------------------------------------------ contexts with a 4-bit cache

def test_cache_format_in_the_config():
    import synth
    for f in (0, hh.HH_WF_Q4G32):
        n, c = 4, 4096
        sizes = [hh.hh_workspace_size(hh.make_config(synth.ONE_B, n, c, 512, weight_format=f + k)) for k in (0, hh.HH_KV_Q4)]
        sh = synth.ONE_B
        kv = n * c * sh.n_layers * sh.n_kv_heads
        extra = 512 * (sh.q_dim + 2 * sh.kv_dim) * 4 + (16 << 20)  # the pass's fp32 rows and split outputs
        assert abs(sizes[0] - sizes[1] - (kv * (256 - 72) - extra)) < 4096
    for bad in (hh.HH_KV_Q4 + 2, 0x200, -1, hh.HH_KV_Q4 + hh.HH_WF_Q4G32):
        cfg = hh.make_config(synth.TINY, 2, 128, weight_format=bad)
        with pytest.raises(hh.HHError) as e:
            hh.hh_workspace_size(cfg)
        assert e.value.status == hh.HH_ERR_UNSUPPORTED
    assert hh.hh_workspace_size(hh.make_config(synth.TINY, 2, 128, weight_format=hh.HH_KV_Q4)) > 0


def test_stream_calls_without_a_context():
    lib = hh.load_library()
    assert lib.hh_fork(None, 0, 1, None) == hh.HH_ERR_INVALID_ARG
    assert lib.hh_truncate(None, 0, 0) == hh.HH_ERR_INVALID_ARG
    assert lib.hh_compact(None, None) == hh.HH_ERR_INVALID_ARG
