"""How calls on an 8-bit cache are cut up, without a GPU."""
import itertools
import os
import shutil
import subprocess

import pytest

from paper_2606_12154_amd import hh

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LDS = 160 << 10


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I" + os.path.join(ROOT, "paper_2606_12154_amd", "csrc"),
                    os.path.join(ROOT, "tests", "kv8_plan_tool.cpp"), "-o", exe], check=True)

    def ask(lines):
        text = "".join(" ".join(map(str, x)) + "\n" for x in lines)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


SEQS, ROWS = (1, 2, 3, 8, 31, 100, 1000), (1, 2, 7, 8, 9, 100, 3000)
HEADS = ((32, 8), (4, 2), (8, 1), (64, 8), (128, 128), (7, 7), (40, 1))


def test_lists(plan):
    """Workspaces have their bound, every split has a pair of blocks, and every number of
    waves is some call's."""
    sizes = [("l", s, s * r, r, h, kv, 8192, n) for s, r, (h, kv), n in itertools.product(
        SEQS, ROWS, HEADS, (1, 2, 3, 16, 33, 128, 1000, 32768))]
    got = plan(sizes)
    for z, (waves, splits, tiles, ws, threads) in zip(sizes, got):
        assert waves in (1, 2, 4, 8) and 1 <= splits <= max(1, min(64, (z[7] + 1) // 2))
        assert tiles == (z[4] // z[5] + 15) // 16 and threads >= z[3] * tiles * z[5] * splits * 64 * waves
        assert ws == (0 if splits == 1 else splits * z[2] * z[4] * 66 * 4) and ws <= hh.HH_KV8_WORKSPACE_MOST
    assert {g[0] for g in got} == {1, 2, 4, 8} and max(g[1] for g in got) > 16


def test_selections(plan):
    """A row's scores fit the threads that search it and their workgroup's LDS; workspaces
    have their bound; every kernel is some call's."""
    sizes = [("s", s, s * r, r, h, kv, p, 0) for s, r, (h, kv), p in itertools.product(
        SEQS, ROWS, HEADS, (1, 2, 63, 64, 65, 512, 513, 576, 577, 1024, 1088, 1089, 2048, 2049, 8192, 8193, 32768))]
    got = plan(sizes)
    for z, (rows, waves, keys, team, chunks, lds, ws, threads) in zip(sizes, got):
        searchers = 64 * waves if team else 64
        each = (-(-z[6] // searchers)) | 1
        assert each <= keys and keys in (9, 17, 33) and 1 <= rows <= min(16, z[3]) and waves <= 16
        assert lds == rows * each * searchers * 4 and lds + 2048 <= LDS
        assert not (team and rows > 1) and (team or not chunks) and (chunks == 0 or chunks * 256 >= z[6])
        assert ws == (0 if not chunks else z[2] * z[5] * (-(-z[6] // 16) * 16) * 4) and ws <= hh.HH_KV8_WORKSPACE_MOST
        assert threads >= -(-z[3] // rows) * z[5] * 64 * waves
    assert {(g[2], g[3], g[4] > 0) for g in got} == {(9, 0, False), (17, 0, False), (33, 0, False), (33, 1, False), (33, 1, True)}


def test_workspaces_of_the_calls():
    A = 1 << 20
    most = 0
    for s, r, (h, kv), pages in itertools.product(SEQS, ROWS, HEADS, (1, 300, 3000, 32768)):
        p = hh.hh_kv8_pool(A, A, 1 << 20, kv, pages, s)
        rows = hh.hh_kv8_rows(A, A, None, s, s * r, r)
        need = (hh.hh_kv8_attention_workspace(p, rows, h), hh.hh_kv8_select_workspace(p, rows, h, 64),
                hh.hh_kv8_attention_blocks_workspace(p, rows, h, 512))
        most = max(most, *need)
    assert (8 << 20) < most <= hh.HH_KV8_WORKSPACE_MOST
