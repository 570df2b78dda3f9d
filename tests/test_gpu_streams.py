"""Forks, cuts and compaction of a context's streams, and contexts whose KV cache is
in 4 bits.

* A forked, cut or compacted stream gives the bits of one that was evaluated by
  itself: the kernels address the cache through the page table, and what they
  compute depends on logical positions only.
* Logits of a 4-bit cache are compared with the fp64 oracle whose cache
  holds the same 4-bit values.  The GPU's keys and values differ from the oracle's
  by their rounding, so now and then a code falls on the other side of a border, a
  whole step away.  fp32: rounding 2^-20 of a value and steps of about a
  third of it put 3e-6 of the codes there, at most about 3 of a prompt's (2 layers x 100 rows x 2
  heads x 128); one moves an attention output by at most w s (w the key's weight,
  near 1/64 in the rows compared; s <= 0.25), through W_o (norm 0.32) and the norm
  (|x| >= 0.4) a logit (rows of E have norm 0.32) by 0.32 (16 / 0.4) (0.32 s w) =
  0.016: typically 16 times less, since that is spread over 256 dimensions, so 1e-4 + 3 x 0.001.
  bf16: fp16 activations put 0.3 % of the codes there, errors of one step at random
  signs, 0.05 of a value's, next to the 0.1 of quantization itself that both sides
  share: no more than the 2e-2 that the fp16 paths are given elsewhere, so 4e-2.
"""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import check_logits
from oracle import kv4
from paper_2606_12154_amd import hh

pytestmark = pytest.mark.gpu
SMALL = synth.ModelShape(2, 512, 8, 2, 64, 1024, 1000, 1e-5, 1e4, True, synth.BF16)
# One layer: (shape, weight format, KV format)
KINDS = {"f32": (synth.TINY, 0, 0), "f32 kv4": (synth.TINY, 0, hh.HH_KV_Q4), "fp16": (SMALL, 0, 0),
         "fp16 kv4": (SMALL, 0, hh.HH_KV_Q4), "q4 kv4": (SMALL, hh.HH_WF_Q4G32, hh.HH_KV_Q4)}


def context(kind, streams=4, context=128, max_prefill=0, seed=3):
    shape, wf, kv = KINDS[kind]
    ctx = hh.Context(hh.make_config(shape, streams, context, max_prefill, weight_format=wf + kv))
    tensors = synth.make_weights(shape, seed, gain_std=0.1)
    ctx.load_weights(tensors)
    return shape, tensors, ctx


@pytest.fixture(scope="module", params=list(KINDS))
def any_ctx(request):
    shape, tensors, ctx = context(request.param, streams=5)
    yield shape, ctx
    ctx.close()


def steps(ctx, streams, feeds):
    """Teacher-forced lockstep steps; logits [steps, streams, vocab]."""
    return np.stack([ctx.decode_step(streams, f, logits=True)[1].copy() for f in feeds])


def feeds_for(shape, n_steps, n, seed):
    return np.random.default_rng(seed).integers(0, shape.vocab, (n_steps, n)).astype(np.int32)


def equal(a, b, what):
    assert np.array_equal(a.view(np.uint32), b.view(np.uint32)), f"{what}: max-abs {np.abs(a - b).max():.3g}"


@pytest.mark.parametrize("n", [1, 15, 16, 17, 48, 61])
def test_fork_gives_the_bits_of_streams_of_their_own(any_ctx, n):
    shape, ctx = any_ctx
    prompt = synth.make_tokens(shape.vocab, n, n)
    f = feeds_for(shape, 20, 3, n)
    ctx.reset()
    for s in (0, 1, 2):
        first, _ = ctx.prefill(s, prompt)
    want = steps(ctx, [0, 1, 2], f)
    ctx.reset()
    ctx.prefill(4, synth.make_tokens(shape.vocab, 33, 1))     # other pages for what follows
    ctx.prefill(1, synth.make_tokens(shape.vocab, 20, 2))     # dropped by the fork
    ctx.prefill(0, prompt)
    ctx.fork(0, [2, 1])
    assert [ctx.length(s) for s in (0, 1, 2)] == [n] * 3
    assert [int(ctx.read_argmax(s, n - 1, 1)[0]) for s in (0, 1, 2)] == [first] * 3
    equal(steps(ctx, [0, 1, 2], f), want, "forked")
    # The pending token is forked too: free-running steps agree.
    ctx.reset()
    ctx.prefill(0, prompt)
    ctx.fork(0, [3])
    for _ in range(4):
        nxt, lg = ctx.decode_step([0, 3], None, logits=True)
        assert nxt[0] == nxt[1]
        equal(lg[0], lg[1], "free-running")


def test_fork_of_an_empty_stream_and_of_forks(any_ctx):
    shape, ctx = any_ctx
    ctx.reset()
    ctx.prefill(1, synth.make_tokens(shape.vocab, 20, 2))
    ctx.fork(0, [1])
    assert ctx.length(1) == 0
    p = synth.make_tokens(shape.vocab, 30, 5)
    f = feeds_for(shape, 40, 4, 6)
    for s in range(4):
        ctx.reset(s)
        ctx.prefill(s, p)
    want = steps(ctx, [0, 1, 2, 3], f)
    ctx.reset()
    ctx.prefill(0, p)
    ctx.fork(0, [1])
    ctx.fork(1, [2, 3])
    got = steps(ctx, [0, 1, 2, 3], f[:10])
    ctx.compact()
    equal(np.concatenate([got, steps(ctx, [0, 1, 2, 3], f[10:])]), want, "forks of forks")


def feed(ctx, s, tokens):
    """Tokens one step at a time: products of one row, whatever follows them (a
    prompt's products are cut up by its number of rows)."""
    for t in tokens:
        _, lg = ctx.decode_step([s], [int(t)], logits=True)
    return lg.copy()


@pytest.mark.parametrize("cut", [1, 16, 20, 32, 39])
def test_truncate(any_ctx, cut):
    """A cut stream continues as one that was never longer, and what it shared
    with another stream stays the other's."""
    shape, ctx = any_ctx
    p = synth.make_tokens(shape.vocab, 40, 7)
    f = feeds_for(shape, 12, 1, cut)
    ctx.reset()
    feed(ctx, 0, p[:cut])
    want = steps(ctx, [0], f)
    ctx.reset(0)
    feed(ctx, 0, p)
    other_want = steps(ctx, [0], f)
    ctx.reset()
    feed(ctx, 0, p)
    ctx.fork(0, [1])
    ctx.truncate(1, cut)
    assert (ctx.length(0), ctx.length(1)) == (40, cut)
    equal(steps(ctx, [1], f), want, "cut stream")
    equal(steps(ctx, [0], f), other_want, "the stream it shared pages with")
    # The pending token is the argmax recorded where the stream ends now.
    ctx.truncate(1, cut + 5)
    _, lg = ctx.decode_step([1], [int(np.argmax(want[4, 0]))], logits=True)
    ctx.truncate(1, cut + 5)
    _, lg2 = ctx.decode_step([1], None, logits=True)
    equal(lg, lg2, "pending token after a cut")
    ctx.truncate(1, 0)
    assert ctx.length(1) == 0
    ctx.truncate(0, ctx.length(0))


def test_cut_inside_a_prompt_has_no_pending_token(any_ctx):
    shape, ctx = any_ctx
    ctx.reset()
    ctx.prefill(0, synth.make_tokens(shape.vocab, 40, 7))
    ctx.fork(0, [2])
    ctx.truncate(0, 30)
    ctx.fork(0, [1])
    for s in (0, 1):
        with pytest.raises(hh.HHError) as e:
            ctx.decode_step([2, s], None)
        assert e.value.status == hh.HH_ERR_INVALID_ARG and ctx.length(s) == 30
    ctx.decode_step([2], None)
    a, lg = ctx.decode_step([0, 1], [7, 7], logits=True)
    equal(lg[0], lg[1], "fork of a cut stream")
    ctx.decode_step([0, 1], None)


def test_prompts_append_to_cut_and_forked_streams(any_ctx):
    shape, ctx = any_ctx
    p, q = synth.make_tokens(shape.vocab, 37, 8), synth.make_tokens(shape.vocab, 21, 9)
    ctx.reset()
    ctx.prefill(0, p)
    _, want = ctx.prefill(0, q, logits="all")
    ctx.reset()
    ctx.prefill(3, p)
    ctx.prefill(3, synth.make_tokens(shape.vocab, 30, 10))
    ctx.fork(3, [0, 2])
    ctx.truncate(0, 37)
    _, got = ctx.prefill(0, q, logits="all")
    equal(got, want, "prompt on a cut stream")
    a = ctx.prefill_batch([2, 0], [q, p])
    ctx.reset()
    assert a.shape == (2,)


def test_compaction_changes_no_result(any_ctx):
    shape, ctx = any_ctx
    lens = [50, 3, 70, 16]
    prompts = [synth.make_tokens(shape.vocab, n, 20 + n) for n in lens]
    f = feeds_for(shape, 24, 4, 11)
    ctx.reset()
    for s, p in enumerate(prompts):
        ctx.prefill(s, p)
    want = steps(ctx, [0, 1, 2, 3], f)
    ctx.reset()
    ctx.prefill(4, synth.make_tokens(shape.vocab, 100, 1))
    for s, p in enumerate(prompts):
        ctx.prefill(s, p)
    ctx.reset(4)
    ctx.fork(0, [4])
    used = sum((n + 15) // 16 for n in lens) + 1   # the fork: three shared pages, one of its own
    assert ctx.compact() == used
    a = steps(ctx, [0, 1, 2, 3], f[:8])
    ctx.reset(4)
    b = steps(ctx, [0, 1, 2, 3], f[8:16])
    in_use = sum((n + 16 + 15) // 16 for n in lens)
    assert ctx.compact() == in_use == ctx.compact()
    c = steps(ctx, [0, 1, 2, 3], f[16:])
    equal(np.concatenate([a, b, c]), want, "compacted")


def test_pages_come_back(any_ctx):
    """Forks and cuts in any order neither lose nor double a page: the pool can
    be filled to its last page afterwards, many times."""
    shape, ctx = any_ctx
    rng = np.random.default_rng(12)
    ctx.reset()
    for i in range(60):
        s = int(rng.integers(0, 5))
        what = rng.integers(0, 4)
        if what == 0:
            n = int(rng.integers(1, 129 - ctx.length(s))) if ctx.length(s) < 128 else 0
            if n:
                ctx.prefill(s, synth.make_tokens(shape.vocab, n, i))
        elif what == 1:
            ctx.fork(s, [t for t in rng.permutation(5)[:int(rng.integers(1, 5))] if t != s] or [(s + 1) % 5])
        elif what == 2:
            ctx.truncate(s, int(rng.integers(0, ctx.length(s) + 1)))
        else:
            ctx.compact()
    ctx.reset()
    assert ctx.compact() == 0
    full = synth.make_tokens(shape.vocab, 128, 13)
    for s in range(5):
        ctx.prefill(s, full)
    assert ctx.compact() == 40


def test_refusals(any_ctx):
    shape, ctx = any_ctx
    ctx.reset()
    ctx.prefill(0, synth.make_tokens(shape.vocab, 20, 2))
    for call in (lambda: ctx.fork(5, [0]), lambda: ctx.fork(-1, [0]), lambda: ctx.fork(0, []), lambda: ctx.fork(0, [0]),
                 lambda: ctx.fork(0, [1, 1]), lambda: ctx.fork(0, [5]), lambda: ctx.fork(0, [1, 2, 3, 4, 1]),
                 lambda: ctx.truncate(5, 0), lambda: ctx.truncate(-1, 0), lambda: ctx.truncate(0, 21),
                 lambda: ctx.truncate(0, -1)):
        with pytest.raises(hh.HHError) as e:
            call()
        assert e.value.status == hh.HH_ERR_INVALID_ARG
    assert ctx.length(0) == 20 and ctx.length(1) == 0


# ------------------------------------------------------------------ the 4-bit cache

class _Rows(list):
    """A layer's cached rows; what is appended is held as its 4-bit values."""

    def __setitem__(self, i, rows):
        n = self[i].shape[0]
        super().__setitem__(i, np.concatenate([rows[:n], kv4.values(rows[n:])]))


def q4_cache(model):
    c = model.new_cache()
    c.k, c.v = _Rows(c.k), _Rows(c.v)
    return c


@pytest.mark.parametrize("kind,tol", [("f32 kv4", 1e-4 + 3e-3), ("fp16 kv4", 4e-2), ("q4 kv4", 4e-2)])
@pytest.mark.parametrize("rows", [0, 40])
def test_logits_against_the_oracle(kind, tol, rows):
    """Prompts (in one pass and in passes of 40 rows), single and lockstep steps."""
    shape, tensors, ctx = context(kind, streams=3, max_prefill=rows)
    w = synth.weights_as_f64(shape, tensors)
    if kind.startswith("q4"):
        w = oracle.q4_model_weights(shape, w)
    model = oracle.Decoder(shape, w)
    prompts = [synth.make_tokens(shape.vocab, n, n) for n in (100, 71, 90)]
    caches, plain = [q4_cache(model) for _ in prompts], model.new_cache()
    refs = [model.forward(p, c) for p, c in zip(prompts, caches)]
    full = model.forward(prompts[0], plain)
    _, got = ctx.prefill(0, prompts[0], logits="all")
    worst = check_logits(got[64:], refs[0][64:], tol, margin=2 * tol, what="prompt")
    # The oracle that keeps its cache in fp64 is further off.
    rms = [float(np.sqrt(np.mean((got[64:] - r[64:]) ** 2))) for r in (refs[0], full)]
    assert rms[0] < 0.7 * rms[1], rms
    nxt = ctx.prefill_batch([1, 2], prompts[1:])
    for i, r in enumerate(refs[1:]):
        if r[-1, np.argsort(r[-1])[-1]] - np.sort(r[-1])[-2] > 2 * tol:
            assert nxt[i] == np.argmax(r[-1])
    toks = feeds_for(shape, 3, 3, 4)
    for f in toks:
        ref = model.decode_batch(caches, f)
        _, lg = ctx.decode_step([0, 1, 2], f, logits=True)
        worst = max(worst, check_logits(lg, ref, tol, margin=2 * tol, what="lockstep"))
    ref = model.decode(caches[1], 5)
    _, lg = ctx.decode_step([1], [5], logits=True)
    worst = max(worst, check_logits(lg[0], ref, tol, margin=2 * tol, what="single"))
    print(f"{kind}: max-abs {worst:.3g}, rms {rms[0]:.3g} against the 4-bit cache, {rms[1]:.3g} against fp64")
    ctx.close()


def test_long_streams_of_a_4_bit_cache():
    """Steps whose attention is split over keys, and graphs of several lengths:
    free-running history equals teacher-forced argmaxes on a second stream."""
    shape, tensors, ctx = context("fp16 kv4", streams=2, context=3000)
    p = synth.make_tokens(shape.vocab, 2040, 3)
    ctx.prefill(0, p)
    ctx.fork(0, [1])
    for i in range(20):
        nxt, _ = ctx.decode_step([0], None)
        prev = int(ctx.read_argmax(0, 2039 + i, 1)[0])
        got, _ = ctx.decode_step([1], [prev])
        assert nxt[0] == got[0], i
    # The same rows as one prompt.
    hist = ctx.read_argmax(0, 2039, 20)
    _, lg = ctx.decode_step([0], None, logits=True)
    ctx.reset(1)
    _, want = ctx.prefill(1, np.concatenate([p, hist, ctx.read_argmax(0, 2059, 1)]), logits="last")
    assert np.abs(lg[0] - want).max() < 4e-2
    ctx.close()


def test_no_single_kernel_step_on_a_4_bit_cache():
    shape, tensors, ctx = context("f32 kv4", streams=2)
    with pytest.raises(hh.HHError) as e:
        hh.hh_decode_step_noalloc(ctx.ctx, 0, 5, None, None)
    assert e.value.status == hh.HH_ERR_UNSUPPORTED
    ctx.close()
