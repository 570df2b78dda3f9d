"""The 1B-class bf16 decoder (d 2048, 32/8 heads, FFN 8192, vocab 128256) with its KV cache in 8 bits against the fp64
oracle whose cache holds the same 8-bit values: a prompt, a batch of prompts, lockstep and single steps.

What the GPU's logits may be off: the fp16 paths' 2e-2 of this model's other tests, and what codes do that fall on the
other side of a border. In terms of D, the rms of what quantization itself does to a row's logits (the distance of the
oracle with the 8-bit cache from the one without): a block's 1,024 values reach 3.3 of their rms and a step is a power of
two, so 3.3 / 127 = 0.026 to 0.052 of the rms, and quantization's error a step / sqrt(12).

One layer. Keys and values come from activations rounded to fp16, 2^-12 / sqrt(3) = 1.4e-4 of a value's rms off, so
0.8 x 1.4e-4 / 0.026 = 4.3e-3 of the codes cross a border at most. In the first row, which attends to itself alone,
2.2 of the 512 values whose errors make D, in any of 150 rows hardly ever ten (a Poisson number of mean 2.2: 6e-5 above
nine): sqrt(10 x 12 / 512) D = 0.48 D, and the largest of 128,256 x 96 logits is 5.4 times the rms: 2.6 D. Over all
rows the mean square is 12 x 4.3e-3 D^2: 0.23 D, 0.4 D with the rows of several. (Another quantization would be
sqrt(2) D off, 7.7 D at the most.)

All 16. Codes that crossed a border move the next layers' values by more than fp16 does, so more cross there, until the
two have nothing of their errors in common: then they are sqrt(2) D from each other, 7.7 D at the most, and each D
from the oracle without quantization.
"""
import numpy as np
import pytest

import oracle
import synth
from paper_2606_12154_amd import hh
from test_gpu_streams_kv8 import q8_cache

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
    ctx = hh.Context(hh.make_config(shape, 4, 512, 128, weight_format=hh.HH_KV_Q8))
    ctx.load_weights(tensors)
    prompts = [synth.make_tokens(shape.vocab, n, n) for n in (96, 33)]
    # The same rows on 8-bit caches and on plain ones.
    caches, plain = ([make() for _ in prompts] for make in (lambda: q8_cache(model), model.new_cache))
    refs, fulls = ([model.forward(p, c) for p, c in zip(prompts, cs)] for cs in (caches, plain))
    times = 2.6 if layers == 1 else 7.7

    def check(got, ref, full, what):
        d = np.sqrt(np.mean(np.square(ref - full), axis=-1))
        err = np.abs(got - ref).max(-1)
        print(f"{layers} layers, {what}: max-abs {err.max():.3g}, rms {rms(got - ref):.3g}; D {rms(d):.3g}, from full {rms(got - full):.3g}")
        assert np.isfinite(got).all()
        assert (err <= 2e-2 + times * d).all(), f"{what}: {(err / (2e-2 + times * d)).max():.3g} of the tolerance"
        return d

    _, got = ctx.prefill(0, prompts[0], logits="all")
    d = rms(check(got, refs[0], fulls[0], "prompt"))
    assert rms(got - refs[0]) <= (0.4 if layers == 1 else 2 ** 0.5) * d + 2e-3
    nxt = ctx.prefill_batch([1, 2], prompts)
    for i, r in enumerate(refs):
        top = np.sort(r[-1])
        if top[-1] - top[-2] > 2 * (2e-2 + times * rms(r[-1] - fulls[i][-1])):
            assert nxt[i] == np.argmax(r[-1])
    for f in np.random.default_rng(4).integers(0, shape.vocab, (2, 2)).astype(np.int32):
        ref, full = model.decode_batch(caches, f), model.decode_batch(plain, f)
        _, lg = ctx.decode_step([1, 2], f, logits=True)
        check(lg, ref, full, "lockstep")
        _, lg = ctx.decode_step([0], [f[0]], logits=True)
        check(lg, ref[:1], full[:1], "single")
    ctx.close()
