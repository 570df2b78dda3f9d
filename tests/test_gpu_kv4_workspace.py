"""Calls of many sizes of hh_kv4_attention in one workspace of the documented bound."""
import numpy as np
import pytest

from paper_2606_12154_amd import hh
from test_gpu_kv4 import attend, check, filled

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_one_workspace_for_streams_that_end():
    """A batch of single tokens that shrinks, and prompt rows, over a table far wider than its sequences."""
    n, pages = 1500, 8192
    c, kv = filled([n], 1, 5, max_pages=pages)
    ws = torch.full((hh.HH_KV4_WORKSPACE_MOST,), 255, dtype=torch.uint8, device="cuda:0")
    needs = set()
    for seqs, rows in ((256, 1), (64, 1), (8, 1), (1, 1), (1, 300), (3, 40), (1, 1200)):
        q = torch.randn(seqs * rows, 4, 64, device="cuda:0")
        out = torch.full_like(q, 9.0)
        first = [n - rows - 3 * (i % 5) for i in range(seqs)]
        r, keep = c.rows(np.arange(seqs + 1) * rows, first, seqs * rows, table_row=np.zeros(seqs))
        needs.add(hh.hh_kv4_attention_workspace(c.desc, r, 4))
        attend(c, r, q, "f32", out, "f32", ws=ws)
        for s in {0, seqs // 2, seqs - 1}:
            at = slice(s * rows, (s + 1) * rows)
            check(out[at].double().cpu().numpy(), q[at].double().cpu().numpy(), *kv[0], 0.125, first[s], "f32")
    assert max(needs) <= hh.HH_KV4_WORKSPACE_MOST and len(needs) > 2
