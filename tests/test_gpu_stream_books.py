"""Prompts, steps, forks, cuts and compaction in any order, by what the streams hold: after each change of
the books a lockstep step of all streams is compared with a second context that evaluated
each stream's tokens as one prompt.

Both contexts' logits are within the tolerance of their kind of the fp64 oracle's (the other tests: 1e-4 for fp32,
2e-2 for fp16 paths; on a 4-bit cache test_gpu_streams.py derives 3.1e-3 and 4e-2), hence within twice that of each
other.  A page of another stream's, or an old one, shows: the test first sees to it that a
stream in which one page's tokens are others differs by more.
"""
import numpy as np
import pytest

from test_gpu_streams import KINDS, context

pytestmark = pytest.mark.gpu
TOL = {"f32": 1e-4, "f32 kv4": 3.1e-3, "fp16": 2e-2, "fp16 kv4": 4e-2, "q4 kv4": 4e-2}
N, CONTEXT = 5, 128


@pytest.mark.parametrize("kind", list(KINDS))
def test_any_order_of_calls(kind):
    shape, tensors, ctx = context(kind, streams=N, context=CONTEXT)
    _, _, other = context(kind, streams=N, context=CONTEXT)
    rng = np.random.default_rng(5)
    held = [np.zeros(0, np.int32) for _ in range(N)]
    tokens = lambda n: rng.integers(0, shape.vocab, n).astype(np.int32)  # noqa: E731
    tol = 2 * TOL[kind]

    def alone(streams, step):
        """Logits of the step, from the tokens alone."""
        other.reset()
        for i, t in enumerate(streams):
            other.prefill(i, t)
        return other.decode_step(list(range(len(streams))), step, logits=True)[1].copy()

    t = tokens(60)
    wrong = t.copy()
    wrong[16:32] = tokens(16)
    a, b = alone([t, wrong], np.array([7, 7], np.int32))
    assert np.abs(a - b).max() > 2 * tol, "a page of other tokens would not show"

    def look(what):
        live = [s for s in range(N) if 0 < len(held[s]) < CONTEXT]
        if not live:
            return
        step = tokens(len(live))
        want = alone([held[s] for s in live], step)
        _, got = ctx.decode_step(live, step, logits=True)
        for s, x, g, w in zip(live, step, got, want):
            assert np.abs(g - w).max() <= tol, f"{what}: stream {s} of {len(held[s])} is {np.abs(g - w).max():.3g} off"
            held[s] = np.append(held[s], x)

    for i in range(70):
        s, what = int(rng.integers(0, N)), int(rng.integers(0, 8))
        n = len(held[s])
        if what <= 2 and n < CONTEXT:
            t = tokens(int(rng.integers(1, min(50, CONTEXT - n) + 1)))
            ctx.prefill(s, t)
            held[s] = np.concatenate([held[s], t])
        elif what <= 4:
            dst = [int(x) for x in rng.permutation(N) if x != s][:int(rng.integers(1, N))]
            ctx.fork(s, dst)
            for x in dst:
                held[x] = held[s].copy()
            look(f"call {i}: fork of {s} to {dst}")
        elif what <= 6:
            m = int(rng.integers(0, n + 1))
            ctx.truncate(s, m)
            held[s] = held[s][:m]
            look(f"call {i}: cut of {s} to {m}")
        else:
            used = ctx.compact()
            assert used <= sum((len(h) + 15) // 16 for h in held)
            look(f"call {i}: compaction")
        assert [ctx.length(x) for x in range(N)] == [len(h) for h in held]
    ctx.close()
    other.close()
