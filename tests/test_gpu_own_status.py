"""A HIP call of the program's own that failed leaves its error on the thread. The calls on
a cache's pages and on streams report their own launches, do their work, and leave that error to the
program."""
import ctypes
from contextlib import contextmanager, nullcontext

import numpy as np
import pytest

import synth
from paper_2606_12154_amd import hh

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@contextmanager
def pending_error():
    """An error of another call's on this thread, still there at the end."""
    torch.cuda.synchronize()
    hh.load_library()
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64" in line)
    hip = ctypes.CDLL(path)
    hip.hipGetLastError.restype = ctypes.c_int
    try:
        assert hip.hipSetDevice(1 << 20) != 0
        yield
        assert hip.hipGetLastError() != 0
    finally:
        hip.hipGetLastError()


def stream():
    return torch.cuda.current_stream().cuda_stream


def test_page_copies_and_compaction():
    pool = torch.randint(0, 256, (2, 12, 1152), dtype=torch.uint8, device="cuda:0")
    want = pool.clone()
    with pending_error():
        hh.hh_kv_copy_pages(pool.data_ptr(), 2, pool.stride(0), 1152, 12, [10, 3], [1, 2], stream())
    want[:, [1, 2]] = want[:, [10, 3]]
    assert torch.equal(pool, want)
    table = torch.tensor([[11, 4]], dtype=torch.int32, device="cuda:0")
    lens = torch.tensor([32], dtype=torch.int32, device="cuda:0")
    live = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(hh.hh_kv_compact_workspace(12), dtype=torch.uint8, device="cuda:0")
    with pending_error():
        hh.hh_kv_compact(pool.data_ptr(), 2, pool.stride(0), 1152, 12, table.data_ptr(), 1, 2, lens.data_ptr(), live.data_ptr(),
                         ws.data_ptr(), ws.numel(), stream())
    want[:, [0, 1]] = want[:, [4, 11]]
    assert torch.equal(pool, want) and table.tolist() == [[1, 0]] and live.item() == 2


@pytest.mark.parametrize("kv", [0, hh.HH_KV_Q4])
def test_forks_cuts_and_compaction_of_streams(kv):
    shape = synth.TINY
    ctx = hh.Context(hh.make_config(shape, 3, 128, weight_format=kv))
    ctx.load_weights(synth.make_weights(shape, 3, gain_std=0.1))
    p = synth.make_tokens(shape.vocab, 40, 7)

    def run(around):
        ctx.reset()
        ctx.prefill(1, p[:20])
        ctx.prefill(0, p)
        with around():
            ctx.fork(0, [1, 2])
        with around():
            ctx.truncate(1, 37)      # copies the shared third page
        ctx.reset(0)
        with around():
            assert ctx.compact() == 4
        return ctx.decode_step([1, 2], [5, 6], logits=True)[1].copy()

    want = run(nullcontext)
    assert np.array_equal(run(pending_error), want)
    ctx.close()


def test_calls_of_a_4_bit_cache():
    n, hkv, hq, pages = 600, 2, 8, 40
    pool = torch.zeros((pages, hkv, 1152), dtype=torch.uint8, device="cuda:0")
    table = torch.arange(pages, dtype=torch.int32, device="cuda:0")
    start, first = (torch.tensor(a, dtype=torch.int32, device="cuda:0") for a in ([0, n], [0]))
    desc = hh.hh_kv4_pool(pool.data_ptr(), table.data_ptr(), pages, hkv, pages, 1)
    rows = hh.hh_kv4_rows(start.data_ptr(), first.data_ptr(), None, 1, n, n)
    last = torch.tensor([n - 1], dtype=torch.int32, device="cuda:0")
    one = hh.hh_kv4_rows(None, last.data_ptr(), None, 1, 1, 1)
    k, v = (torch.randn(n, hkv, 64, device="cuda:0") for _ in "kv")
    q = torch.randn(1, hq, 64, device="cuda:0")
    ws = torch.zeros(hh.hh_kv4_attention_workspace(desc, one, hq), dtype=torch.uint8, device="cuda:0")

    def run(around):
        pool.zero_()
        back, out = [torch.full_like(k, 9.0) for _ in "kv"], torch.full_like(q, 9.0)
        with around():
            hh.hh_kv4_append(desc, rows, k.data_ptr(), v.data_ptr(), hh.HH_F32, 128, 128, None, 0, stream())
        with around():
            hh.hh_kv4_read(desc, rows, back[0].data_ptr(), back[1].data_ptr(), hh.HH_F32, 128, 128, stream())
        with around():
            hh.hh_kv4_attention(desc, one, q.data_ptr(), hh.HH_F32, hq * 64, hq, 0.125, None, 0, out.data_ptr(), hh.HH_F32,
                                hq * 64, ws.data_ptr() or None, ws.numel(), stream())
        return [pool.clone(), *back, out]

    for a, b in zip(run(nullcontext), run(pending_error)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("wf", [0, hh.HH_KV_Q4])
def test_steps_and_prompts(wf):
    """Steps work beside the error; a prompt reports it with nothing done."""
    shape = synth.TINY
    ctx = hh.Context(hh.make_config(shape, 3, 128, weight_format=wf))
    ctx.load_weights(synth.make_weights(shape, 3, gain_std=0.1))
    p = synth.make_tokens(shape.vocab, 24, 7)

    def run(around):
        ctx.reset()
        for s in range(3):
            ctx.prefill(s, p[s:])
        out = []
        for i in range(10):  # across a page's end
            with around():
                out.append(ctx.decode_step([0], [int(p[i])], logits=True)[1].copy())
            with around():
                out.append(ctx.decode_step([1, 2], [int(p[i])] * 2, logits=True)[1].copy())
            with around():
                out.append(ctx.decode_step([1, 2], None, logits=True)[1].copy())
        return out

    for a, b in zip(run(nullcontext), run(pending_error)):
        assert np.array_equal(a, b)
    ctx.reset()
    _, want = ctx.prefill(0, p, logits="all")
    for n in (24, 3):  # with new pages, and without
        ctx.reset()
        if n == 3:
            ctx.prefill(0, p[:21])
        hip_error = pytest.raises(hh.HHError)
        with pytest.raises(AssertionError), pending_error():  # (it is taken)
            with hip_error as e:
                ctx.prefill(0, p[24 - n:])
        assert e.value.status == hh.HH_ERR_HIP and ctx.length(0) == 24 - n
        _, got = ctx.prefill(0, p[24 - n:], logits="all")
        if n == 24:
            assert np.array_equal(got, want)
        assert ctx.length(0) == 24
    ctx.close()


def test_probe_and_quantizer():
    x = torch.randn(8, 64, device="cuda:0").bfloat16()
    got, want = (torch.zeros(8, 36, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    hh.hh_q4g32_quantize(x.data_ptr(), 8, 64, want.data_ptr(), stream())
    with pending_error():
        hh.hh_q4g32_quantize(x.data_ptr(), 8, 64, got.data_ptr(), stream())
    assert torch.equal(got, want)
    with pending_error():
        hh.hh_read_probe(x.data_ptr(), x.numel() * 2, stream())
