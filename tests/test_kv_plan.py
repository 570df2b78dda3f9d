"""How the attention over a 4-bit cache is cut up, without a GPU."""
import itertools

import pytest

from paper_2606_12154_amd import hh

A = 1 << 20  # an aligned address that no call here may read


def need(seqs, rows, max_pages, heads=32, kv_heads=8, max_rows=None):
    pool = hh.hh_kv4_pool(A, A, max_pages * seqs, kv_heads, max_pages, seqs)
    r = hh.hh_kv4_rows(A, A, None, seqs, seqs * rows, max_rows or rows)
    return hh.hh_kv4_attention_workspace(pool, r, heads)


def test_workspace_has_a_bound():
    """One allocation serves every call: sizes from a token to long prompts, any page table."""
    most = 0
    for seqs, rows, pages in itertools.product((1, 2, 3, 8, 31, 32, 64, 128, 256, 1000), (1, 2, 5, 16, 40, 150, 300, 1000, 8192),
                                               (1, 19, 63, 320, 2048, 8192, 65536)):
        for heads, kv in ((32, 8), (4, 2), (8, 1), (64, 8), (128, 128), (7, 7)):
            most = max(most, need(seqs, rows, pages, heads, kv))
    assert (8 << 20) < most <= hh.HH_KV4_WORKSPACE_MOST


@pytest.mark.parametrize("heads,kv_heads", [(1 << 25, 1), ((1 << 25) + 1024, 1024), (1 << 30, 2)])
def test_heads_past_32_bit_offsets_are_refused(heads, kv_heads):
    """A row's elements are counted in 32 bits."""
    with pytest.raises(hh.HHError) as e:
        need(1, 1, 1, heads, kv_heads)
    assert e.value.status == hh.HH_ERR_UNSUPPORTED
    pool = hh.hh_kv4_pool(A, A, 1, kv_heads, 1, 1)
    with pytest.raises(hh.HHError) as e:
        hh.hh_kv4_attention(pool, hh.hh_kv4_rows(None, A, None, 1, 1, 1), A, hh.HH_F16, heads * 64, heads, 1.0, None, 0, A,
                            hh.HH_F16, heads * 64, A, 1 << 30, None)
    assert e.value.status == hh.HH_ERR_UNSUPPORTED
