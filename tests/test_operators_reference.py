"""The 64-bit forms that the operators are tested against, themselves held against differences of their
own values and against closed forms (no GPU)."""
import numpy as np
import pytest

import operators_reference as ref


def direction(f, x, g, rng, step=1e-5):
    """(f(x + e d) - f(x - e d)) / 2 e against <g, d> along a random d."""
    d = rng.standard_normal(x.shape)
    rise = (f(x + step * d) - f(x - step * d)) / (2 * step)
    want = float((g * d).sum())
    assert abs(rise - want) <= 1e-6 * (1 + float(np.abs(g * d).sum()))


@pytest.mark.parametrize("causal,pre,cap,bias", [(False, False, 0.0, False), (True, False, 0.0, True), (True, True, 3.0, True)])
def test_attention_gradients_are_differences(causal, pre, cap, bias):
    rng = np.random.default_rng(3)
    B, T, Hq, Hkv, D = 2, 13, 4, 2, 5
    reset, valid, seq_id, n = ref.flags(rng, B, T, 5)
    prefix = rng.integers(0, 5, n) if pre else None
    see = ref.visible(reset, valid, seq_id, causal, prefix)
    slopes = rng.random(Hq) if bias else None
    q, k, v = (rng.standard_normal((B, T, h, D)) for h in (Hq, Hkv, Hkv))
    w = rng.standard_normal((B, T, Hq, D))
    r = ref.attention(q, k, v, see, 0.6, cap, slopes, "f32", w)
    loss = lambda q, k, v: float((ref.attention(q, k, v, see, 0.6, cap, slopes, "f32")["out"][0] * w).sum())
    direction(lambda x: loss(x, k, v), q, r["dq"][0], rng)
    direction(lambda x: loss(q, x, v), k, r["dk"][0], rng)
    direction(lambda x: loss(q, k, x), v, r["dv"][0], rng)


@pytest.mark.parametrize("state", [False, True])
def test_gated_gradients_are_differences(state):
    rng = np.random.default_rng(4)
    B, T, D = 3, 17, 4
    reset, valid, _, _ = ref.flags(rng, B, T, 6)
    reset[:, 0] = 0
    gate, x, w = rng.random((B, T, D)), rng.standard_normal((B, T, D)), rng.standard_normal((B, T, D))
    h0 = rng.standard_normal((B, D)) if state else None
    ws = rng.standard_normal((B, D))
    r = ref.gated(gate, x, reset, valid, h0, "f32", w, ws)

    def loss(gate, x, h0):
        y = ref.gated(gate, x, reset, valid, h0, "f32")
        return float((y["h"][0] * w).sum() + (y["state"][0] * ws).sum())
    direction(lambda z: loss(z, x, h0), gate, r["dgate"][0], rng)
    direction(lambda z: loss(gate, z, h0), x, r["dx"][0], rng)
    if state:
        direction(lambda z: loss(gate, x, z), h0, r["dh0"][0], rng)


def test_gated_constant_gate_is_the_decayed_sum():
    T = 9
    r = ref.gated(np.full((1, T, 1), 0.5), np.ones((1, T, 1)), np.zeros((1, T), np.uint8), np.ones((1, T), np.uint8), None, "f32")
    assert np.allclose(r["h"][0][0, :, 0], 2 - 0.5 ** np.arange(T), rtol=1e-14)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_keeps_lengths_and_turns_back(layout):
    rng = np.random.default_rng(5)
    x, pos = rng.standard_normal((2, 7, 3, 10)), rng.integers(-1, 1000, (2, 7))
    freq = 10.0 ** -np.arange(3)
    y, _ = ref.rotary(x, pos, freq, layout, 1.0, False)
    back, _ = ref.rotary(y, pos, freq, layout, 1.0, True)
    live = pos >= 0
    assert np.allclose(back[live], x[live], atol=1e-12) and not back[~live].any()
    assert np.allclose((y[live] ** 2).sum(-1), (x[live] ** 2).sum(-1))
    assert np.array_equal(y[live][..., 6:], x[live][..., 6:])
