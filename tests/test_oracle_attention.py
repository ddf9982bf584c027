"""The oracle's masked transformer stage: its gradients against central
differences, and the unmasked special case against the plain attention."""
import numpy as np
import pytest

import synth
from oracle import stages

ATTENTION = {
    "causal": synth.AttentionSpec(causal=True, rotary_dim=8),
    "all": synth.AttentionSpec(causal=True, cap=3.0, slopes=True, rotary_dim=4, rotary_layout="interleaved",
                               rotary_scaling="parts", rotary_factor=4.0, rotary_original_length=8),
    "ntk": synth.AttentionSpec(rotary_dim=16, rotary_scaling="ntk", rotary_factor=2.0),
}


def _spec(attention):
    return synth.StageSpec("transformer", "bf16", "none", 0, 1, 2, 1, (64, 4, 64, 8), 1e-3, 0.9, attention=attention)


@pytest.mark.parametrize("name", list(ATTENTION))
def test_gradients_match_differences(name):
    spec = _spec(ATTENTION[name])
    g = np.random.default_rng(5)
    masks = {"documents": np.array([[0, 0, 0, 1, 1, 1, 0, 0], [4] * 8], np.int32),
             "kv_lengths": np.array([8, 6], np.int32)}
    if spec.attention.causal:
        masks["prefix"] = np.array([2, 5], np.int32)
    W = synth.initial_params(spec).astype(np.float64)
    x, dy = g.normal(size=spec.input_shape()), g.normal(size=spec.output_shape())

    def value(W, x):
        return float((stages.forward(spec, stages.unpack(spec, W), x, exact=True, masks=masks)[0] * dy).sum())

    P = stages.unpack(spec, W)
    _, _, st = stages.forward(spec, P, x, exact=True, masks=masks)
    dx, grads = stages.backward(spec, P, st, dy, exact=True, masks=masks)
    for at, grad in ((0, stages.pack(spec, grads)), (1, dx)):
        d = g.normal(size=(W, x)[at].shape)
        h = 1e-6
        hi = value(W + h * d, x) if at == 0 else value(W, x + h * d)
        lo = value(W - h * d, x) if at == 0 else value(W, x - h * d)
        want = (hi - lo) / (2 * h)
        assert abs(float((grad * d).sum()) - want) <= 1e-5 * max(1.0, abs(want))


def test_an_attention_without_options_is_the_plain_one():
    spec, plain = _spec(synth.AttentionSpec()), _spec(None)
    P = stages.unpack(spec, synth.initial_params(spec))
    x = np.random.default_rng(1).normal(size=spec.input_shape())
    y0, _, s0 = stages.forward(plain, P, x)
    y1, _, s1 = stages.forward(spec, P, x)
    assert np.array_equal(y0, y1)
    dy = np.random.default_rng(2).normal(size=spec.output_shape())
    (a, ga), (b, gb) = stages.backward(plain, P, s0, dy), stages.backward(spec, P, s1, dy)
    assert np.allclose(a, b, rtol=1e-12, atol=1e-12) and all(np.allclose(ga[n], gb[n]) for n in ga)
