"""The 64-bit forms that the norms, the short convolution and the selective scan are tested against, themselves held against differences
of their own values and closed forms (no GPU)."""
import numpy as np
import pytest

import operators_reference as ref
import state_space_reference as ssr
from test_operators_reference import direction


@pytest.mark.parametrize("center", [False, True])
def test_norm_gradients_are_differences(center):
    rng = np.random.default_rng(1)
    rows, D = 7, 11
    s, dy, ds = (rng.standard_normal((rows, D)) for _ in range(3))
    w, b = rng.standard_normal(D), rng.standard_normal(D)
    live = np.arange(rows) != 3
    r = ssr.norm(s, w, b, live, 1e-3, center, "f32", dy, ds)
    loss = lambda s, w, b: float((ssr.norm(s, w, b, live, 1e-3, center, "f32")["out"][0] * dy).sum() + (s * ds)[live].sum())
    direction(lambda t: loss(t, w, b), s, r["dx"][0], rng)
    direction(lambda t: loss(s, t, b), w, r["dweight"][0], rng)
    direction(lambda t: loss(s, w, t), b, r["dbias"][0], rng)


def test_norm_has_the_size_it_should():
    s = np.random.default_rng(2).standard_normal((5, 64)) * 3 + 2
    y = ssr.norm(s, None, None, np.ones(5, bool), 0.0, True, "f32")["out"][0]
    assert np.allclose(y.mean(1), 0, atol=1e-12) and np.allclose((y * y).mean(1), 1)
    y = ssr.norm(s, None, None, np.ones(5, bool), 0.0, False, "f32")["out"][0]
    assert np.allclose(y, s / np.sqrt((s * s).mean(1, keepdims=True)))


@pytest.mark.parametrize("T,K,silu,state", [(17, 4, True, False), (17, 3, False, True), (2, 4, True, True), (1, 8, True, True), (9, 1, True, False)])
def test_conv_gradients_are_differences(T, K, silu, state):
    rng = np.random.default_rng([T, K])
    B, D = 3, 4
    reset, valid, _, _ = ref.flags(rng, B, T, 6)
    if state:
        reset[:, 0] = 0
    x, dy = (rng.standard_normal((B, T, D)) for _ in range(2))
    w, b = rng.standard_normal((D, K)), rng.standard_normal(D)
    s0, ds = (rng.standard_normal((B, K - 1, D)) if state else None for _ in range(2))
    r = ssr.conv(x, w, b, reset, valid, silu, s0, "f32", dy, ds)

    def loss(x, w, b, s0):
        y = ssr.conv(x, w, b, reset, valid, silu, s0, "f32")
        return float((y["out"][0] * dy).sum() + (0 if ds is None else (y["state"][0] * ds).sum()))
    direction(lambda t: loss(t, w, b, s0), x, r["dx"][0], rng)
    direction(lambda t: loss(x, t, b, s0), w, r["dweight"][0], rng)
    direction(lambda t: loss(x, w, t, s0), b, r["dbias"][0], rng)
    if state:
        direction(lambda t: loss(x, w, b, t), s0, r["dstate_in"][0], rng)


def test_conv_of_whole_sequences_by_numpy():
    rng = np.random.default_rng(3)
    B, T, D, K = 2, 30, 3, 4
    reset, valid, _, _ = ref.flags(rng, B, T, 7)
    x, w = rng.standard_normal((B, T, D)), rng.standard_normal((D, K))
    y = ssr.conv(x, w, None, reset, valid, False, None, "f32")["out"][0]
    for b in range(B):
        for f, e in ref.segments(reset[b], valid[b]):
            for d in range(D):
                assert np.allclose(y[b, f:e, d], np.convolve(x[b, f:e, d], w[d, ::-1])[:e - f])


@pytest.mark.parametrize("softplus,gated,state", [(True, True, True), (False, False, False), (True, False, True)])
def test_scan_gradients_are_differences(softplus, gated, state):
    rng = np.random.default_rng(4)
    B, T, D, N, G = 2, 12, 6, 3, 2
    reset, valid, _, _ = ref.flags(rng, B, T, 5)
    if state:
        reset[:, 0] = 0
    names = ["x", "dt", "rate", "b", "c", "skip", "z", "bias", "h0"]
    args = dict(x=rng.standard_normal((B, T, D)), dt=0.1 + 0.3 * rng.random((B, T, D)), rate=-rng.random((D, N)) * 3,
                b=rng.standard_normal((B, T, G, N)), c=rng.standard_normal((B, T, G, N)), skip=rng.standard_normal(D),
                z=rng.standard_normal((B, T, D)) if gated else None, bias=0.1 * rng.standard_normal(D),
                h0=rng.standard_normal((B, D, N)) if state else None)
    dy, ds = rng.standard_normal((B, T, D)), rng.standard_normal((B, D, N))

    def call(dy=None, ds=None, **kw):
        a = {**args, **kw}
        return ssr.scan(a["x"], a["dt"], a["rate"], a["b"], a["c"], reset, valid, a["skip"], a["z"], a["bias"], softplus, a["h0"], "f32", dy, ds)
    r = call(dy, ds)

    def loss(**kw):
        y = call(**kw)
        return float((y["out"][0] * dy).sum() + (y["state"][0] * ds).sum())
    for name, grad in zip(names, ("dx", "ddt", "drate", "db", "dc", "dskip", "dz", "ddt_bias", "dh0")):
        if args[name] is not None:
            direction(lambda t: loss(**{name: t}), args[name], r[grad][0], rng)


def test_scan_of_one_state_is_the_decayed_sum():
    """A rate of ln(1/2) and steps of 1 halve the state with every frame."""
    T = 9
    one = np.ones((1, T, 1))
    r = ssr.scan(one, one, np.full((1, 1), np.log(0.5)), one[..., None], one[..., None], np.zeros((1, T), np.uint8), np.ones((1, T), np.uint8),
                 None, None, None, False, None, "f32")
    assert np.allclose(r["out"][0][0, :, 0], 2 - 0.5 ** np.arange(T), rtol=1e-14)
