"""A paged step's attention keeps as many bits as the prefill's: the same prompt through both, with values that cancel.

Tokens come in pairs of opposite embeddings, so that their values v and -v add up to nothing and a row's result is what the probabilities differ by: keys are short (gain 2^-6), all
scores within a few hundredths of each other, and what is left is about 2^-6 of the values.  A rounding of the probabilities to 16 bits (up to 2^-18 of
one, 2^-19.5 root mean square) comes out as about 2^-13.5 of it.

Tolerance.  Both calls round a result to two bf16 planes and the rows behind the layer to two more, each up to 2^-18 of its value, and add in float32 (2^-24 a step, over sums
that the pairs keep as small as the result); keys, values and queries are rounded alike by both.  Even if all four erred fully and the same way, a logit were off by
4 x 2^-18 = 2^-16 of the root of its terms' squares, which the largest of 300 exceeds: 2^-16 of the largest logit."""
import numpy as np
import pytest

import dmtd_inputs as di
import paper_2510_11958_amd as pkg
from parity_util import engine_config, norm_err

V, WIDTH, N = 300, 256, 512


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 2, 64), (3, 3, 128)])
@pytest.mark.parametrize("chunks", [(N,), (N - 2, 2), (N - 64, 57, 6, 1)])
def test_values_that_cancel(heads, chunks):
    nh, nkv, hd = heads
    sh = di.ModelShape(1, WIDTH, nh, nkv, hd, 64, V, tied_embeddings=False)
    rng = np.random.RandomState(hd + nh)
    half = rng.normal(size=(V // 2, WIDTH)) * 0.02
    one, zero = np.ones(WIDTH), np.zeros((64, WIDTH))

    def matrix(n, k, scale):
        return rng.normal(size=(n, k)) * scale / np.sqrt(k)

    parts = [np.concatenate([half, -half]), one, matrix(nh * hd, WIDTH, 1), matrix(nkv * hd, WIDTH, 1), matrix(nkv * hd, WIDTH, 1), np.ones(hd), np.full(hd, 2.0 ** -6),
             matrix(WIDTH, nh * hd, 256), one, zero, zero, np.zeros((WIDTH, 64)), one, matrix(V, WIDTH, 1)]
    blob = di.f32_to_bf16_bits(np.concatenate([np.asarray(p, np.float32).ravel() for p in parts]))
    assert blob.size == di.blob_elems(sh)
    first = rng.randint(0, V // 2, N // 2)
    prompt = np.stack([first, first + V // 2], 1).reshape(1, N).astype(np.int32)
    eng = pkg.Engine(engine_config(sh, N + 2), blob)
    eng.prefill(prompt)
    ref = eng.logits()[0].astype(np.float64)
    assert np.isfinite(ref).all()
    eng.reset()
    eng.paged_begin(16)
    at = 0
    for n in chunks:
        eng.paged_step([0], [prompt[0, at:at + n]], [1], 1)
        at += n
    err = norm_err(eng.logits()[0], ref)
    print("error", err * 2 ** 16, "x 2^-16")
    assert err < 2.0 ** -16
