"""Page copies and compaction on the GPU against numpy (exact: bytes)."""
import numpy as np
import pytest

from paper_2606_12154_amd import hh

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def stream():
    return torch.cuda.current_stream().cuda_stream


def random_pool(layers, pages, size, gap, seed):
    """Layers `gap` bytes further apart than their pages reach."""
    rng = np.random.default_rng(seed)
    a = rng.integers(0, 256, (layers, pages * size + gap), dtype=np.uint8)
    return a, torch.from_numpy(a.copy()).to("cuda:0")


@pytest.mark.parametrize("layers,size,gap,n,sources", [(1, 16, 0, 1, 1), (2, 1152, 0, 30, 30), (3, 9216, 4096, 61, 7),
                                                       (16, 4112, 16, 490, 490), (1, 131072, 0, 3, 1), (2, 32, 0, 1200, 5)])
def test_copies(layers, size, gap, n, sources):
    pages = 2 * n + 5
    a, d = random_pool(layers, pages, size, gap, n)
    order = np.random.default_rng(n).permutation(pages)
    dst, src = order[:n], order[n:n + sources][np.arange(n) % sources]
    hh.hh_kv_copy_pages(d.data_ptr(), layers, pages * size + gap, size, pages, src, dst, stream())
    p = a[:, :pages * size].reshape(layers, pages, size)
    p[:, dst] = p[:, src].copy()
    a[:, :pages * size] = p.reshape(layers, -1)
    assert np.array_equal(d.cpu().numpy(), a)


def reference(pool, table, lengths, size):
    """pool [layers, pages, size] and table compacted in place; returns the live count."""
    pages = pool.shape[1]
    held = np.arange(table.shape[1])[None] < np.clip(-(-lengths // 16), 0, table.shape[1])[:, None]
    real = held & (table >= 0) & (table < pages)
    used = np.zeros(pages, bool)
    used[table[real]] = True
    live = int(used.sum())
    src, dst = np.flatnonzero(used[live:]) + live, np.flatnonzero(~used[:live])
    pool[:, dst] = pool[:, src].copy()
    to = np.arange(pages)
    to[src] = dst
    table[real] = to[table[real]]
    return live


@pytest.mark.parametrize("layers,pages,size,rows,cols,fill,seed", [
    (1, 1, 16, 1, 1, 1.0, 0), (2, 7, 1152, 3, 4, 0.5, 1), (1, 33, 4096, 4, 9, 0.9, 2), (3, 1000, 9216, 17, 60, 0.5, 3),
    (1, 1000, 64, 17, 60, 0.0, 4), (2, 4097, 128, 40, 110, 1.0, 5), (1, 70000, 16, 300, 200, 0.7, 6),
    (1, 1 << 20, 16, 64, 9000, 0.4, 7)])
def test_compaction(layers, pages, size, rows, cols, fill, seed):
    rng = np.random.default_rng(seed)
    a, d = random_pool(layers, pages, size, 32, seed)
    ids = rng.permutation(pages)
    table = np.full((rows, cols), 1 << 30, np.int32)  # entries past a length: anything
    lengths = np.zeros(rows, np.int32)
    at = 0
    for r in range(rows):
        n = min(int(rng.integers(0, cols + 1)), int(fill * pages) - at)
        n = max(n, 0)
        table[r, :n] = ids[at:at + n]
        at += n
        if r and n and rng.random() < 0.5:  # a shared first page
            table[r, 0] = table[0, 0] if lengths[0] else table[r, 0]
        lengths[r] = max(0, 16 * n - int(rng.integers(0, 16)))
    if rows > 2:
        lengths[2] = -5                      # no positions
        table[1, 0] = -1                     # names no page
    d_table, d_len = torch.from_numpy(table.copy()).to("cuda:0"), torch.from_numpy(lengths).to("cuda:0")
    live = torch.full((1,), -1, dtype=torch.int32, device="cuda:0")
    need = hh.hh_kv_compact_workspace(pages)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda:0")
    call = (d.data_ptr(), layers, pages * size + 32, size, pages, d_table.data_ptr(), rows, cols, d_len.data_ptr(),
            live.data_ptr(), ws.data_ptr(), need)
    hh.hh_kv_compact(*call, stream())
    p = a[:, :pages * size].reshape(layers, pages, size)
    want = reference(p, table, lengths, size)
    a[:, :pages * size] = p.reshape(layers, -1)
    assert live.item() == want
    assert np.array_equal(d_table.cpu().numpy(), table)
    assert np.array_equal(d.cpu().numpy(), a)
    # A compact pool stays as it is.
    hh.hh_kv_compact(*call, stream())
    assert live.item() == want and np.array_equal(d_table.cpu().numpy(), table) and np.array_equal(d.cpu().numpy(), a)


def test_captured_copy_and_compaction():
    a, d = random_pool(2, 40, 1152, 0, 3)
    table = torch.tensor([[30, 3, 39], [7, 8, 0]], dtype=torch.int32, device="cuda:0")
    first, lengths = table.clone(), torch.tensor([48, 20], dtype=torch.int32, device="cuda:0")
    live = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(hh.hh_kv_compact_workspace(40), dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()

    def body():
        hh.hh_kv_copy_pages(d.data_ptr(), 2, 40 * 1152, 1152, 40, [30, 3], [20, 21], stream())
        hh.hh_kv_compact(d.data_ptr(), 2, 40 * 1152, 1152, 40, table.data_ptr(), 2, 3, lengths.data_ptr(), live.data_ptr(),
                         ws.data_ptr(), ws.numel(), stream())

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    for i in range(4):
        d.random_(0, 256)
        lengths.copy_(torch.tensor([48 - 16 * (i % 3), 20 + i], dtype=torch.int32))
        p, t = d.cpu().numpy().reshape(2, 40, 1152).copy(), first.cpu().numpy().copy()
        table.copy_(first)
        graph.replay()
        torch.cuda.synchronize()
        p[:, [20, 21]] = p[:, [30, 3]].copy()
        want = reference(p, t, lengths.cpu().numpy(), 1152)
        assert live.item() == want and np.array_equal(table.cpu().numpy(), t), i
        assert np.array_equal(d.cpu().numpy().reshape(2, 40, 1152), p), i
