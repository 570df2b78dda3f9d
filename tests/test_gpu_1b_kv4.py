"""The 1B-class bf16 decoder (d 2048, 32/8 heads, FFN 8192, vocab 128256) with its KV cache in 4 bits against the fp64
oracle whose cache holds 4-bit values too: a prompt, a batch of prompts, lockstep and single steps.

What the GPU's logits may be off: the fp16 paths' 2e-2 of this model's other tests, and what codes do that fall on the
other side of a border. In terms of D, the rms of what quantization itself does to a row's logits (the distance of the
oracle with the 4-bit cache from the one without): a step is about a third of a value's rms, quantization's error a
step / sqrt(12).

One layer. Keys and values come from activations rounded to fp16, 2^-12 / sqrt(3) = 1.4e-4 of a value's rms off, so
0.8 x 1.4e-4 / 0.33 = 3.4e-4 of the codes cross a border: of a row's 1,024 a third of one on average, of 96 rows' hardly
ever five in one row. In the first row, which attends to itself alone, a value is 1 of 512 whose errors make D, so a step
in one is sqrt(12 / 512) D = 0.15 D, in four 0.3 D; the largest of 128,256 x 96 logits is 5.4 times the rms: 1.7 D. Over
all rows the mean square is 12 x 3.4e-4 D^2, 0.06 D; 0.2 D with the rare rows of several. (Other quantization would be D off
and 5.4 D.)

All 16. Codes that crossed a border move the next layers' values by far more than fp16 does, so more cross there: their
share grows to where the first row's errors are only half D (0.075 of x a layer; e' ^2 = e^2 + 29 e 0.075^2 from
e = 1.4e-4 passes 0.075 in four layers). No bound of an element follows, but the two share what did not cross: over the
later rows, which average many keys, they are nearer to each other than either is to the oracle without
quantization, 0.7 of it at most, and as far from that one as each other.
"""
import numpy as np
import pytest

import oracle
import synth
from paper_2606_12154_amd import hh
from test_gpu_streams import q4_cache

pytestmark = pytest.mark.gpu


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


@pytest.mark.parametrize("layers", [1, 16])
def test_prompts_and_steps(layers):
    one = synth.ONE_B
    shape = synth.ModelShape(layers, one.d_model, one.n_heads, one.n_kv_heads, one.head_dim, one.ffn_dim, one.vocab,
                             one.rms_eps, one.rope_theta, one.tied, one.dtype)
    tensors = synth.make_weights(shape, 1)
    model = oracle.Decoder(shape, synth.weights_as_f64(shape, tensors))
    ctx = hh.Context(hh.make_config(shape, 4, 512, 128, weight_format=hh.HH_KV_Q4))
    ctx.load_weights(tensors)
    prompts = [synth.make_tokens(shape.vocab, n, n) for n in (96, 33)]
    # The same rows on 4-bit caches and on plain ones.
    caches, plain = ([make() for _ in prompts] for make in (lambda: q4_cache(model), model.new_cache))
    refs, fulls = ([model.forward(p, c) for p, c in zip(prompts, cs)] for cs in (caches, plain))

    def check(got, ref, full, what):
        d = np.sqrt(np.mean(np.square(ref - full), axis=-1))
        err = np.abs(got - ref).max(-1)
        print(f"{layers} layers, {what}: max-abs {err.max():.3g}, rms {rms(got - ref):.3g}; D {rms(d):.3g}")
        assert np.isfinite(got).all()
        if layers == 1:
            assert (err <= 2e-2 + 1.7 * d).all(), f"{what}: {(err / (2e-2 + 1.7 * d)).max():.3g} of the tolerance"

    _, got = ctx.prefill(0, prompts[0], logits="all")
    check(got, refs[0], fulls[0], "prompt")
    near, far, d = rms(got[48:] - refs[0][48:]), rms(got[48:] - fulls[0][48:]), rms(refs[0][48:] - fulls[0][48:])
    if layers == 1:
        assert rms(got - refs[0]) <= 0.2 * rms(refs[0] - fulls[0]) + 2e-3
    assert near <= 0.7 * d and abs(far / d - 1) <= 0.25, (near, far, d)
    nxt = ctx.prefill_batch([1, 2], prompts)
    for i, r in enumerate(refs):
        top = np.sort(r[-1])
        if layers == 1 and top[-1] - top[-2] > 2 * (2e-2 + 1.7 * rms(r[-1] - fulls[i][-1])):
            assert nxt[i] == np.argmax(r[-1])
    for f in np.random.default_rng(4).integers(0, shape.vocab, (2, 2)).astype(np.int32):
        ref, full = model.decode_batch(caches, f), model.decode_batch(plain, f)
        _, lg = ctx.decode_step([1, 2], f, logits=True)
        check(lg, ref, full, "lockstep")
        assert rms(lg - ref) <= 0.7 * rms(ref - full)
        _, lg = ctx.decode_step([0], [f[0]], logits=True)
        check(lg, ref[:1], full[:1], "single")
        assert rms(lg - ref[:1]) <= 0.7 * rms(ref[:1] - full[:1])
    ctx.close()
