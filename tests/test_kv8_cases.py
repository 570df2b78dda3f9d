"""What the cases of test_gpu_kv8_forms.py reach, without a GPU."""
import os
import shutil
import subprocess

import pytest

import kv4_cases
from kv8_cases import LISTS, LONG, sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    tmp, out = tmp_path_factory.mktemp("plan"), {}
    for tool in ("kv4_plan_tool", "kv8_plan_tool"):
        exe = str(tmp / tool)
        subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2606_12154_amd", "csrc"),
                        os.path.join(ROOT, "tests", tool + ".cpp"), "-o", exe], check=True)
        out[tool[:3]] = lambda lines, exe=exe: [tuple(map(int, l.split())) for l in subprocess.run(
            [exe], input="".join(" ".join(map(str, x)) + "\n" for x in lines), capture_output=True, text=True, check=True).stdout.splitlines()]
    return out


def kernel(z, plan):
    """The kernel that a call over all keys takes (cut up as the 4-bit cache's), and the most steps of a wave."""
    (_, _, max_rows, hq, hkv, pages), (nq, _, waves, splits) = z, plan
    columns = max_rows * (hq // hkv)
    few = nq == 1 and columns <= 16
    pairs = (pages + 1) // 2
    steps = -(-(-(-pairs // splits)) // waves)
    return ("few", 2 if columns <= 8 else 1, waves) if few else ("tiles", nq, 4), splits > 1, steps


def test_cases_reach_every_kernel(plans):
    names = list(kv4_cases.CASES)
    got = {kernel(z, p)[:2] for z, p in zip(map(kv4_cases.sizes, names), plans["kv4"]([kv4_cases.sizes(n) for n in names]))}
    kernels = [("few", p, w) for p in (1, 2) for w in (4, 8)] + [("tiles", nq, 4) for nq in (1, 2, 4)]
    assert {(k, s) for k in kernels for s in (False, True)} - got <= {(("tiles", 1, 4), True)}, got


def test_long_cases_read_their_page_ids_anew(plans):
    z = [sizes(*c) for c in LONG.values()]
    got = [kernel(a, p) for a, p in zip(z, plans["kv4"](z))]
    assert all(steps > 64 for _, _, steps in got), dict(zip(LONG, got))
    assert {k[:2] for k, _, _ in got} >= {("few", 1), ("few", 2), ("tiles", 2), ("tiles", 4)}, got


def test_lists_are_cut_up_every_way(plans):
    z = [("l", 1, r, r, hkv * g, hkv, (r + f + 15) // 16, n) for r, f, hkv, g, n in LISTS.values()]
    got = dict(zip(LISTS, plans["kv8"](z)))
    assert {w for w, *_ in got.values()} == {1, 2, 4, 8}, got
    assert {s > 1 for _, s, *_ in got.values()} == {False, True} and max(s for _, s, *_ in got.values()) > 16
    steps = {name: -(-(-(-((LISTS[name][4] + 1) // 2) // s)) // w) for name, (w, s, *_) in got.items()}
    assert sum(n > 64 for n in steps.values()) >= 4, steps
    assert {t for _, _, t, *_ in got.values()} >= {1, 3}
