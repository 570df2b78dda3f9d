"""How the attention over a 4-bit cache is cut up, without a GPU."""
import itertools
import os
import shutil
import subprocess

import pytest

from kv4_cases import CASES, sizes
from paper_2606_12154_amd import hh

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

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


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2606_12154_amd", "csrc"),
                    os.path.join(ROOT, "tests", "kv4_plan_tool.cpp"), "-o", exe], check=True)

    def ask(sizes):
        text = "".join(" ".join(map(str, s)) + "\n" for s in sizes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_cases_reach_every_kernel(plan):
    """Column tiles, pages side by side and waves, each with one split and with several, and both
    kernels that join splits: what kv4_cases.py lists, and the GPU tests compare, takes them all."""
    names = list(CASES)
    got = dict(zip(names, plan([sizes(n) for n in names])))
    reached = {(*p[:3], p[3] > 1) for p in got.values()}
    shapes = [(1, 1, 4), (1, 1, 8), (1, 0, 4), (1, 0, 8), (2, 0, 4), (4, 0, 4)]
    assert reached == {(*s, several) for s in shapes for several in (False, True)}, got
    outs = {n: sizes(n)[1] * sizes(n)[3] for n in names}
    joins = {p[3] > 16 or (p[3] > 4 and outs[n] <= 512) for n, p in got.items() if p[3] > 1}
    assert joins == {False, True}


def test_no_other_kernel_is_chosen(plan):
    """Over the sizes of a server: nothing but the kernels of the cases."""
    ask = [(q, q * r, r, hkv * g, hkv, p) for q, r, p, (hkv, g) in
           itertools.product((1, 4, 32, 200), (1, 2, 4, 9, 40, 300, 5000), (1, 20, 300, 8192), ((8, 4), (1, 8), (2, 2), (40, 1)))]
    for nq, packed, waves, splits in plan(ask):
        assert (nq, packed, waves) in {(1, 1, 4), (1, 1, 8), (1, 0, 4), (1, 0, 8), (2, 0, 4), (4, 0, 4)} and 1 <= splits <= 64
