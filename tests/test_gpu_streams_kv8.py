"""Contexts whose KV cache is in 8 bits: forks, cuts, compaction, prompts in passes and
steps.

Logits are compared with the fp64 oracle whose cache holds the same 8-bit values,
appended in the same calls (a page's codes are rounded again as its scale grows).  The GPU's
keys and values differ from the oracle's by their rounding, so that now and then a code falls on
the other side of a border, a whole step away.  fp32: rounding is 2^-20 of a value, values
are about 40 steps, so 40 x 2^-19 = 8e-5 of the codes: at most about 4 of a prompt's (2 layers x
100 rows x 2 heads x 128).  One moves an attention output by at most w s (w the key's weight, near
1/64 in the rows compared; s <= 1/32), through W_o (norm 0.32) and the norm (|x| >= 0.4) a logit
(rows of E have norm 0.32) by 0.32 (16 / 0.4) (0.32 s w) = 0.002: typically 16 times less, since
that is spread over 256 dimensions, so 1e-4 + 4 x 1.3e-4 < 1e-3.  bf16: fp16 activations
put (40 x 2^-11) 2 % of the codes there, errors of a step at random signs, 0.14 of its rms beside
the 0.29 of quantization itself that both sides share and that is a tenth of the 4-bit cache's:
below the 2e-2 that the fp16 paths are given elsewhere, so 3e-2 with them.
"""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import check_logits
from oracle import kv8
from paper_2606_12154_amd import hh

pytestmark = pytest.mark.gpu
SMALL = synth.ModelShape(2, 512, 8, 2, 64, 1024, 1000, 1e-5, 1e4, True, synth.BF16)
KINDS = {"f32": (synth.TINY, 0, 1e-3), "fp16": (SMALL, 0, 3e-2), "q4": (SMALL, hh.HH_WF_Q4G32, 3e-2)}


def context(kind, streams=4, context=128, max_prefill=0):
    shape, wf, tol = KINDS[kind]
    ctx = hh.Context(hh.make_config(shape, streams, context, max_prefill, weight_format=wf + hh.HH_KV_Q8))
    tensors = synth.make_weights(shape, 3, gain_std=0.1)
    ctx.load_weights(tensors)
    w = synth.weights_as_f64(shape, tensors)
    return shape, ctx, oracle.Decoder(shape, oracle.q4_model_weights(shape, w) if wf else w), tol


class _Rows(list):
    """A layer's cached rows; what is appended is held as its 8-bit values."""

    def __init__(self, rows, pages=16):
        super().__init__(rows)
        self.held = [kv8.Cache(1, pages, r.shape[1]) for r in rows]

    def __setitem__(self, i, rows):
        n = self[i].shape[0]
        if len(rows) > n:
            self.held[i].append(0, n, rows[n:], np.zeros_like(rows[n:]))
        super().__setitem__(i, self.held[i].values(0, len(rows))[0])

    def cut(self, n):
        for i in range(len(self)):
            super().__setitem__(i, self[i][:n])


def q8_cache(model):
    c = model.new_cache()
    c.k, c.v = _Rows(c.k), _Rows(c.v)
    return c


def in_parts(model, cache, prompt, sizes):
    """A prompt's logits, evaluated in parts as the passes of a call are."""
    at = np.cumsum([0] + list(sizes))
    return np.concatenate([model.forward(prompt[a:b], cache) for a, b in zip(at, at[1:])])


def passes(lens, cap):
    """The parts of each of several prompts that share passes of `cap` rows."""
    out, room = [], cap
    for n in lens:
        out.append([])
        while n:
            take = min(n, room)
            out[-1].append(take)
            n, room = n - take, room - take or cap
    return out


def feeds_for(shape, n_steps, n, seed):
    return np.random.default_rng(seed).integers(0, shape.vocab, (n_steps, n)).astype(np.int32)


def steps(ctx, streams, feeds):
    return np.stack([ctx.decode_step(streams, f, logits=True)[1].copy() for f in feeds])


def equal(a, b, what):
    assert np.array_equal(a.view(np.uint32), b.view(np.uint32)), f"{what}: max-abs {np.abs(a - b).max():.3g}"


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("rows", [0, 40])
def test_logits_against_the_oracle(kind, rows):
    """Prompts (in one pass and in passes of 40 rows), single and lockstep steps."""
    shape, ctx, model, tol = context(kind, streams=3, max_prefill=rows)
    prompts = [synth.make_tokens(shape.vocab, n, n) for n in (100, 71, 90)]
    cap = rows or 128
    caches = [q8_cache(model) for _ in prompts]
    parts = passes([100], cap) + passes([71, 90], cap)
    refs = [in_parts(model, c, p, x) for p, c, x in zip(prompts, caches, parts)]
    _, got = ctx.prefill(0, prompts[0], logits="all")
    check_logits(got[64:], refs[0][64:], tol, margin=2 * tol, what="prompt")
    nxt = ctx.prefill_batch([1, 2], prompts[1:])
    for i, r in enumerate(refs[1:]):
        if np.sort(r[-1])[-1] - np.sort(r[-1])[-2] > 2 * tol:
            assert nxt[i] == np.argmax(r[-1])
    for f in feeds_for(shape, 12, 3, 4):
        ref = model.decode_batch(caches, f)
        _, lg = ctx.decode_step([0, 1, 2], f, logits=True)
        check_logits(lg, ref, tol, margin=2 * tol, what="lockstep")
    ref = model.decode(caches[1], 5)
    _, lg = ctx.decode_step([1], [5], logits=True)
    check_logits(lg[0], ref, tol, margin=2 * tol, what="single")
    ctx.close()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("n", [1, 15, 16, 17, 61])
def test_fork_gives_the_bits_of_streams_of_their_own(kind, n):
    shape, ctx, _, _ = context(kind)
    prompt = synth.make_tokens(shape.vocab, n, n)
    f = feeds_for(shape, 20, 3, n)
    for s in (0, 1, 2):
        ctx.prefill(s, prompt)
    want = steps(ctx, [0, 1, 2], f)
    ctx.reset()
    ctx.prefill(3, synth.make_tokens(shape.vocab, 33, 1))
    ctx.prefill(0, prompt)
    ctx.fork(0, [2, 1])
    got = steps(ctx, [0, 1, 2], f[:9])
    ctx.reset(3)
    ctx.compact()
    equal(np.concatenate([got, steps(ctx, [0, 1, 2], f[9:])]), want, "forked and compacted")
    ctx.close()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("cut", [1, 16, 20, 32, 39])
def test_truncate(kind, cut):
    """A cut stream goes on as the oracle's (its last page keeps its scale), what it
    shared with another stream stays the other's; cut between pages it has the bits of
    a stream that was never longer."""
    shape, ctx, model, tol = context(kind)
    p = synth.make_tokens(shape.vocab, 40, 7)
    f = feeds_for(shape, 12, 1, cut)

    def feed(s, tokens):
        for t in tokens:
            ctx.decode_step([s], [int(t)])

    feed(0, p[:cut])
    short = steps(ctx, [0], f)
    ctx.reset(0)
    feed(0, p)
    other_want = steps(ctx, [0], f)
    ctx.reset()
    feed(0, p)
    ctx.fork(0, [1])
    ctx.truncate(1, cut)
    cache = q8_cache(model)
    for t in p:
        model.decode(cache, int(t))
    cache.k.cut(cut)
    cache.v.cut(cut)
    got = steps(ctx, [1], f)
    want = np.stack([model.decode(cache, int(t[0])) for t in f])
    if cut % 16 == 0:
        equal(got, short, "cut between pages")
    # (Rows of few keys: a code's step counts for as much more as a key's weight, 64 / cut.)
    check_logits(got[:, 0], want, max(tol, 1e-4 + 5.2e-4 * 64 / cut if kind == "f32" else 0), margin=10 * tol, what="cut stream")
    equal(steps(ctx, [0], f), other_want, "the stream it shared pages with")
    ctx.close()


def test_long_streams():
    """Steps whose attention is split over keys, and graphs of several lengths:
    free-running history equals teacher-forced argmaxes on a second stream."""
    shape, ctx, _, _ = context("fp16", streams=2, context=3000)
    p = synth.make_tokens(shape.vocab, 2040, 3)
    ctx.prefill(0, p)
    ctx.fork(0, [1])
    for i in range(20):
        nxt, _ = ctx.decode_step([0], None)
        prev = int(ctx.read_argmax(0, 2039 + i, 1)[0])
        got, _ = ctx.decode_step([1], [prev])
        assert nxt[0] == got[0], i
    hist = ctx.read_argmax(0, 2039, 20)
    _, lg = ctx.decode_step([0], None, logits=True)
    ctx.reset(1)
    _, want = ctx.prefill(1, np.concatenate([p, hist, ctx.read_argmax(0, 2059, 1)]), logits="last")
    assert np.abs(lg[0] - want).max() < 4e-2
    ctx.close()


def test_pages_come_back():
    """Forks and cuts in any order neither lose nor double a page."""
    shape, ctx, _, _ = context("f32", streams=5)
    rng = np.random.default_rng(12)
    for i in range(60):
        s, what = int(rng.integers(0, 5)), rng.integers(0, 4)
        if what == 0 and ctx.length(s) < 128:
            ctx.prefill(s, synth.make_tokens(shape.vocab, int(rng.integers(1, 129 - ctx.length(s))), i))
        elif what == 1:
            ctx.fork(s, [t for t in rng.permutation(5)[:int(rng.integers(1, 5))] if t != s] or [(s + 1) % 5])
        elif what == 2:
            ctx.truncate(s, int(rng.integers(0, ctx.length(s) + 1)))
        else:
            ctx.compact()
    ctx.reset()
    assert ctx.compact() == 0
    for s in range(5):
        ctx.prefill(s, synth.make_tokens(shape.vocab, 128, 13))
    assert ctx.compact() == 40
    ctx.close()


def test_no_single_kernel_step():
    shape, ctx, _, _ = context("f32", streams=2)
    with pytest.raises(hh.HHError) as e:
        hh.hh_decode_step_noalloc(ctx.ctx, 0, 5, None, None)
    assert e.value.status == hh.HH_ERR_UNSUPPORTED
    ctx.close()
