"""The model's operators at the edges of what their callers may do, on the GPU."""
import os
import sys

import numpy as np
import pytest
import torch

import operators_reference as ref
from gpu_util import binding, to_dev

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


# rows that are no whole number of a lane's elements: their last lane and its neighbour meet at the borders of wavefronts and workgroups
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("B,T,D", [(130, 1, 9), (200, 1, 37), (130, 1, 81), (130, 1, 257), (130, 1, 1025), (2, 1, 2049), (130, 8, 9),
                                   (130, 3, 81), (300, 1, 3), (130, 2, 40)])
def test_gated_state_in_place(B, T, D, dtype):
    """A state that is advanced where it lies, and its gradient, bit for bit as from one buffer to another."""
    print(f"gated in place B={B} T={T} D={D} {dtype}", flush=True)
    bl = binding()
    rng = np.random.default_rng([B, T, D])
    gate, x, w = (ref.draw(rng, (B, T, D), dtype).cuda() for _ in range(3))
    gate = gate.sigmoid()
    reset, valid = (to_dev((rng.random((B, T)) < p).astype(np.uint8)) for p in (0.1, 0.9))
    state, dstate = (torch.from_numpy(rng.standard_normal((B, D)).astype(np.float32)).cuda() for _ in range(2))
    h, last = bl.bload_gated_scan(gate, x, reset, valid, h0=state)
    dgate, dx, dh0 = bl.bload_gated_scan_backward(w, gate, h, reset, valid, h0=state, dstate=dstate)
    here, there = state.clone(), dstate.clone()
    h_in_place, same = bl.bload_gated_scan(gate, x, reset, valid, h0=here, state=here)
    assert same is here and torch.equal(h_in_place, h) and torch.equal(here, last)
    grads = torch.empty_like(dgate), torch.empty_like(dx), there
    bl.bload_gated_scan_backward(w, gate, h, reset, valid, h0=state, dstate=there, grads=grads)
    assert torch.equal(grads[0], dgate) and torch.equal(grads[1], dx) and torch.equal(there, dh0)


def capped(dtype, cap, size, decode=False):
    """Attention of one sequence with scores of some `size`, capped: the result, lse and gradients against 64 bits.  A computed score
    is off by the products' (D + 4) 2^-24 of its terms' sizes and by 2^-18 of itself; everything else as in operators_reference."""
    bl = binding()
    B, T, H, D = 1, 150, 2, 64
    rng = np.random.default_rng([T, int(size)])
    q, k, v, g = (ref.draw(rng, (B, T, H, D), dtype) for _ in range(4))
    scale = size / 8.0                                      # (q.k has a deviation of 8)
    see = np.ones((B, T, T), bool)
    want = {}
    Q, K, V, G = (np.moveaxis(ref.wide(t), 2, 1) for t in (q, k, v, g))
    s0 = scale * Q @ K.swapaxes(2, 3)
    off = (D + 4) * ref.U32 * scale * (np.abs(Q) @ np.abs(K).swapaxes(2, 3)) + 2.0 ** -18 * np.abs(s0)
    t = np.tanh(s0 / cap)
    s, keep = cap * t, 1 - t * t
    # (a small x leaves keep as it is, but for a rounding; the derivative of keep by s0 is below 1 / cap)
    keep_off = 2 * off / cap + 4 * ref.U32
    m = s.max(3, keepdims=True)
    p = np.exp(s - m)
    total = p.sum(3, keepdims=True)
    p /= total
    u, z = ref.half_step(dtype), ref.tiny(dtype)
    d = 2.5 * (off + 8 * ref.U32 * (np.abs(s) + np.abs(m) + 1)).max(3, keepdims=True) + (T + 8) * ref.U32
    out, lse = p @ V, np.log(total) + m
    out_off = (d + u) * (p @ np.abs(V)) + z * np.abs(V).sum(2, keepdims=True)
    want["out"] = out, out_off + u * np.abs(out) + z
    want["lse"] = lse[..., 0], (d + 4 * ref.U32 * (np.abs(lse) + 1))[..., 0]
    d = 2 * d + 8 * ref.U32 * (np.abs(lse) + 1)              # the backward pass takes p from the stored lse
    dp, dp_off = G @ V.swapaxes(2, 3), (D + 2) * ref.U32 * (np.abs(G) @ np.abs(V).swapaxes(2, 3))
    delta = (G * out).sum(3, keepdims=True)
    delta_off = (np.abs(G) * (out_off + (2 * u * u + D * ref.U32) * np.abs(out) + z)).sum(3, keepdims=True)
    ds = p * (dp - delta) * keep
    ds_off = (d + u) * np.abs(ds) + p * (dp_off + delta_off + keep_off * np.abs(dp - delta)) + z
    for name, a, a_off, x in (("dq", ds, ds_off, K), ("dk", ds.swapaxes(2, 3), ds_off.swapaxes(2, 3), Q)):
        value = scale * a @ x
        want[name] = value, scale * (a_off + 2 * T * ref.U32 * np.abs(a)) @ np.abs(x) + u * np.abs(value) + z
    dv = p.swapaxes(2, 3) @ G
    want["dv"] = dv, ((d + u + 2 * T * ref.U32) * p + z).swapaxes(2, 3) @ np.abs(G) + u * np.abs(dv) + z
    dq, dk, dv, dg = (x.cuda() for x in (q, k, v, g))
    one = torch.ones((B, T), dtype=torch.uint8, device="cuda")
    mask = bl.bload_segment_mask(torch.zeros_like(one), one, causal=False)
    kw = dict(scale=scale, cap=cap)
    y, saved = bl.bload_segment_attention(dq, dk, dv, mask, training=True, **kw)
    got = [y, *bl.bload_segment_attention_backward(dg, dq, dk, dv, y, saved, mask, **kw)]
    for name, x in zip(("out", "dq", "dk", "dv"), got):
        ref.assert_close(x.permute(0, 2, 1, 3), *want[name], f"{name} {dtype} cap {cap} scores of {size}")
    ref.assert_close(saved.lse, *want["lse"], f"lse {dtype} cap {cap} scores of {size}")
    table = [to_dev(np.array([n], np.int32)) for n in (0, 0, T)]
    for row in (0, T - 1):
        x = bl.bload_segment_attention_decode(dq[:, row], dk, dv, *table, **kw)
        ref.assert_close(x[0], want["out"][0][0, :, row], want["out"][1][0, :, row], f"single query {dtype} cap {cap} scores of {size}")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("cap,size", [(1e3, 1), (1e4, 1), (1e5, 1), (1e6, 1), (1e9, 1), (1e30, 1), (3e38, 1), (200.0, 30), (1e5, 30), (1e-3, 1), (1e-42, 1)])
def test_large_and_small_caps(cap, size, dtype):
    """A cap far above the scores leaves them as they are; one far below leaves all alike."""
    print(f"cap {cap} scores of {size} {dtype}", flush=True)
    capped(dtype, cap, size)


def gradients(T, dtype, starts, causal, q, k, v, g, where=None):
    """dq, dk and dv of one block of sequences that begin at `starts`, with one head of keys and a scale of 1, against 64 bits, with
    bounds that hold over the whole range of a type: a gradient of a score, p (dp - delta), keeps half a step of the type however small dout is.
    (float16 packs it as a multiple, the row's largest above 2^6 and float16's smallest normal number 2^-14: the step holds down to 2^-20 of
    the row's largest, where these inputs lie; the bound's 2^-37 of the largest dp - delta is stricter than what holds below.)
    A probability keeps it down to 2^-37.  where: the slots to compare."""
    bl = binding()
    H, D, scale = q.shape[2], q.shape[3], 1.0
    at = np.arange(T)
    seq = np.searchsorted(starts, at, side="right")
    see = (seq[:, None] == seq) & ((at[:, None] >= at) | (not causal))
    Q, K, V, G = (np.moveaxis(ref.wide(t), 2, 1)[0] for t in (q, k, v, g))
    u, z = ref.half_step(dtype), ref.tiny(dtype)
    z_ds = 2.0 ** -37 if dtype == "f16" else 0.0
    s = scale * Q @ K.swapaxes(1, 2)
    off = (D + 4) * ref.U32 * scale * (np.abs(Q) @ np.abs(K).swapaxes(1, 2)) + 4 * ref.U32 * (np.abs(s) + 1)
    m = np.where(see, s, -np.inf).max(2, keepdims=True)
    p = np.where(see, np.exp(s - m), 0)
    total = p.sum(2, keepdims=True)
    p /= total
    lse = np.log(total) + m
    d = 2.5 * np.where(see, off + 4 * ref.U32 * np.abs(s - m), 0).max(2, keepdims=True) + (T + 8) * ref.U32
    out = p @ V
    out_off = (d + u) * (p @ np.abs(V)) + z * (see @ np.abs(V))
    d = 2 * d + 12 * ref.U32 * (np.abs(lse) + 1)             # the backward pass takes p from the stored lse
    dp, dp_off = G @ V.swapaxes(1, 2), (D + 2) * ref.U32 * (np.abs(G) @ np.abs(V).swapaxes(1, 2))
    delta = (G * out).sum(2, keepdims=True)
    delta_off = (np.abs(G) * (out_off + (2 * u * u + D * ref.U32) * np.abs(out) + z)).sum(2, keepdims=True)
    ds = p * (dp - delta)
    ds_off = (d + u) * np.abs(ds) + p * (dp_off + delta_off)
    size = np.where(see, np.abs(dp - delta) + dp_off + delta_off, 0)
    dq = scale * ds @ K
    dq_off = scale * (ds_off + 2 * T * ref.U32 * np.abs(ds) + z_ds * see * size.max(2, keepdims=True)) @ np.abs(K)
    t = lambda x: x.swapaxes(1, 2)
    dk = (scale * t(ds) @ Q).sum(0)
    dk_off = (scale * t(ds_off + 2 * H * T * ref.U32 * np.abs(ds) + z_ds * see * size.max((0, 1))) @ np.abs(Q)).sum(0)
    dv = (t(p) @ G).sum(0)
    dv_off = (t((d + u + 2 * H * T * ref.U32) * p + z_ds * see) @ np.abs(G)).sum(0)
    want = [(x, x_off + u * np.abs(x) + z) for x, x_off in ((dq, dq_off), (dk, dk_off), (dv, dv_off))]
    dq, dk, dv, dg = (x.cuda() for x in (q, k, v, g))
    reset = to_dev(np.isin(at, starts).astype(np.uint8)[None])
    mask = bl.bload_segment_mask(reset, torch.ones_like(reset), causal=causal)
    y, saved = bl.bload_segment_attention(dq, dk, dv, mask, scale=scale, training=True)
    got = bl.bload_segment_attention_backward(dg, dq, dk, dv, y, saved, mask, scale=scale)
    live = np.ones(T, bool) if where is None else where
    for name, x, (value, bound) in zip(("dq", "dk", "dv"), got, want):
        x = np.moveaxis(ref.wide(x), 2, 1)[0]
        value, bound = (y if y.ndim == 3 else y[None] for y in (value, bound))
        # a value that the type cannot hold is infinite in it
        x = np.where((np.abs(value) + bound > torch.finfo(ref.TORCH[dtype]).max) & (x == np.copysign(np.inf, value)), value, x)
        ref.assert_close(x[:, live], value[:, live], bound[:, live], f"{name} T={T} {dtype}")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("gain", [1e-6, 1e-5, 1e-3, 1.0, 1e4])
@pytest.mark.parametrize("causal,D", [(False, 64), (True, 40), (False, 128)])
def test_gradients_of_small_and_large_dout(causal, D, gain, dtype):
    """One long sequence whose values are its keys, so that dq is dout times their spread, at any size of dout."""
    print(f"gradients D={D} {dtype} causal {causal} dout of {gain}", flush=True)
    T, H = 1500, 2
    rng = np.random.default_rng([T, D])
    q, k, g = (ref.draw(rng, (1, T, h, D), "f32") for h in (H, 1, H))
    q, k, g = (x.to(ref.TORCH[dtype]) for x in (q / D, k, g * gain))
    gradients(T, dtype, [0], causal, q, k, k, g)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("rise", [6.0, -6.0])
def test_gradients_of_sizes_that_change(rise, causal, dtype):
    """dout, or values, that grow or shrink by a factor of 10^6 along a sequence."""
    T, H, D = 700, 2, 64
    rng = np.random.default_rng(T)
    q, k, v, g = (ref.draw(rng, (1, T, h, D), "f32") for h in (H, 1, 1, H))
    slope = torch.from_numpy(10.0 ** (rise * (np.arange(T) / T - 0.5))).float()[None, :, None, None]
    half = slope.abs() ** 0.5
    for x, y in ((v, g * slope), (v * half, g), (v * half, g * half.flip(1))):
        gradients(T, dtype, [0], causal, *(t.to(ref.TORCH[dtype]) for t in (q / 8, k, x, y)))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_beside_a_sequence_of_large_ones(causal, dtype):
    """The largest gradients of a neighbour in the block leave small ones as they are."""
    T, H, D = 300, 2, 64
    rng = np.random.default_rng(T)
    q, k, g = (ref.draw(rng, (1, T, h, D), "f32") for h in (H, 1, H))
    starts = [0, 45, 90, 200]
    loud = (np.arange(T) >= 45) & (np.arange(T) < 90)
    g = g * torch.from_numpy(np.where(loud, 1e4, 1e-6)).float()[None, :, None, None]
    q, k, g = (x.to(ref.TORCH[dtype]) for x in (q / 8, k, g))
    gradients(T, dtype, starts, causal, q, k, k, g, ~loud)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (40, 1, 37), (2, 2, 128)])
@pytest.mark.parametrize("T,n", [(200, 1), (200, 31), (200, 32), (200, 33), (200, 130), (2000, 33), (2000, 1999)])
def test_single_query_with_an_infinite_value(T, n, Hq, Hkv, D, dtype):
    """A value that is seen and infinite: infinite in the result, where it lies, whatever tile or share it ends (T decides on the shares)."""
    print(f"single query T={T} n={n} Hq={Hq} Hkv={Hkv} D={D} {dtype}", flush=True)
    bl = binding()
    rng = np.random.default_rng([T, n, Hq, D])
    q, k, v = (ref.draw(rng, (1, t, h, D), dtype).cuda() for t, h in ((1, Hq), (T, Hkv), (T, Hkv)))
    table = [to_dev(np.array([x], np.int32)) for x in (0, T - n, n)]
    one = torch.ones((1, n), dtype=torch.uint8, device="cuda")
    mask = bl.bload_segment_mask(torch.zeros_like(one), one, causal=False)
    clean = bl.bload_segment_attention_decode(q[0], k, v, *table)
    assert torch.isfinite(clean).all()
    for at, value in ((T - 1, float("inf")), (T - n, float("-inf")), (T - 1 - n // 2, float("nan"))):
        v2 = v.clone()
        v2[0, at, :, D // 2] = value
        got = bl.bload_segment_attention_decode(q[0], k, v2, *table)
        wide = torch.cat([torch.zeros((1, n - 1, Hq, D), dtype=q.dtype, device="cuda"), q], 1)
        whole = bl.bload_segment_attention(wide, k[:, T - n:], v2[:, T - n:], mask)[0, -1:]
        want = torch.full((1, Hq), value, dtype=q.dtype, device="cuda")
        for x in (got, whole):
            assert torch.equal(x[:, :, D // 2].nan_to_num(nan=5.0), want.nan_to_num(nan=5.0)), f"value {value} at {at}"
        rest = torch.arange(D, device="cuda") != D // 2
        # (the same sums in another order, and probabilities that are not rounded: a few steps of the type)
        assert ((got - clean)[:, :, rest].float().abs() <= 8 * ref.half_step(dtype) * (clean[:, :, rest].float().abs() + 1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n", [(200, 7), (200, 150), (2000, 1999)])
def test_values_near_the_largest(T, n, dtype):
    """Sums of them leave float32, their mean does not."""
    bl = binding()
    rng = np.random.default_rng([T, n])
    big = 0.9 * float(torch.finfo(ref.TORCH[dtype]).max)
    q, k = (ref.draw(rng, (1, t, 2, 32), dtype).cuda() for t in (1, T))
    v = torch.full((1, T, 2, 32), big, dtype=ref.TORCH[dtype], device="cuda")
    v[..., 1::2] *= -1
    table = [to_dev(np.array([x], np.int32)) for x in (0, T - n, n)]
    got = bl.bload_segment_attention_decode(q[0], k, v, *table)
    one = torch.ones((1, n), dtype=torch.uint8, device="cuda")
    mask = bl.bload_segment_mask(torch.zeros_like(one), one, causal=False)
    whole = bl.bload_segment_attention(k[:, T - n:], k[:, T - n:], v[:, T - n:], mask)
    # a mean of equal values: the weights' sum is off by n + 8 roundings, the result by one of the type
    off = (n + 8) * ref.U32 + 2 * ref.half_step(dtype)
    for x, y in ((got, v[0, :1]), (whole, v[:, :n])):
        assert torch.isfinite(x).all() and ((x.double() / y.double() - 1).abs() <= off).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D", [64, 90, 128])
@pytest.mark.parametrize("at", [0, 63, 200, 389])
def test_one_element_that_is_not_finite(at, D, dtype):
    """Causally, in one of two sequences: in v or dout it reaches its own element of what depends on it, in q or k all of it, and
    nothing else changes but for the rounding of what is computed another way."""
    print(f"one element at {at} D={D} {dtype}", flush=True)
    bl = binding()
    T, Hq, Hkv, d = 400, 4, 2, D // 3
    rng = np.random.default_rng([at, D])
    q, k, v, g = (ref.draw(rng, (1, T, h, D), dtype).cuda() for h in (Hq, Hkv, Hkv, Hq))
    reset = torch.zeros((1, T), dtype=torch.uint8, device="cuda")
    reset[0, 390] = 1
    mask = bl.bload_segment_mask(reset, torch.ones_like(reset))

    def both(q, k, v, g):
        out, saved = bl.bload_segment_attention(q, k, v, mask, training=True)
        return [t[0] for t in (out, *bl.bload_segment_attention_backward(g, q, k, v, out, saved, mask))]
    clean = both(q, k, v, g)
    own = torch.arange(T, device="cuda")
    behind, front, here = (own >= at) & (own < 390), own <= at, own == at
    heads = {Hq: slice(0, Hq // Hkv), Hkv: slice(0, 1)}                 # those of the first head of keys

    def check(tensors, lost):
        """lost: which elements of out, dq, dk, dv (rows, elements) of the first head of keys are not finite"""
        for i, (got, want) in enumerate(zip(both(*tensors), clean)):
            gone = torch.zeros_like(got, dtype=torch.bool)
            if lost[i] is not None:
                rows, elements = lost[i]
                part = gone[:, heads[got.shape[1]] if lost[4] is None else lost[4] if got.shape[1] == Hq else slice(0, 1)]
                part[rows] = elements
            name = f"{('out', 'dq', 'dk', 'dv')[i]}"
            assert not torch.isfinite(got[gone]).any(), name
            assert torch.isfinite(got[~gone]).all(), name
            # either way is within the bound of the other tests; a few steps of the type of sums of some 400 terms
            off = 32 * ref.half_step(dtype) * (want.float().abs() + 1)
            assert ((got.float() - want.float()).abs() <= off)[~gone].all(), name
    every = torch.ones(D, dtype=torch.bool, device="cuda")
    one = torch.arange(D, device="cuda") == d
    for value in (float("inf"), float("nan")):
        x = v.clone()
        x[0, at, 0, d] = value
        # (a query that sees it has no delta, so it has no dq, and the keys that it sees have no dk)
        check((q, k, x, g), ((behind, one), (behind, every), (own < 390, every), None, None))
        x = g.clone()
        x[0, at, 0, d] = value
        check((q, k, v, x), (None, (here, every), (front, every), (front, one), slice(0, 1)))
    x = q.clone()
    x[0, at, 0, d] = float("nan")
    check((x, k, v, g), ((here, every), (here, every), (front, every), (front, every), slice(0, 1)))


def test_example_takes_the_gradient_of_a_sum():
    """It is one element with strides of 0; the gradients are those of ones."""
    import packed_layer
    bl = binding()
    B, T, H, D = 2, 40, 2, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    one = torch.ones((B, T), dtype=torch.uint8, device="cuda")
    mask, reset = bl.bload_segment_mask(torch.zeros_like(one), one), torch.zeros_like(one)
    at = torch.arange(B * T, dtype=torch.int32, device="cuda").view(B, T)
    freq = bl.bload_rotary_frequencies(D).cuda()
    new = lambda *shape: torch.rand(shape, device="cuda", generator=g).requires_grad_()
    x, q, k, v, gate, y = new(B, T, H, D), new(B, T, H, D), new(B, T, H, D), new(B, T, H, D), new(B, T, D), new(B, T, D)
    for f, leaves in ((lambda: packed_layer.Rotary.apply(x, at, freq), (x,)),
                      (lambda: packed_layer.SegmentAttention.apply(q, k, v, mask), (q, k, v)),
                      (lambda: packed_layer.GatedScan.apply(gate, y, reset, one), (gate, y))):
        out = f()
        want = torch.autograd.grad(out, leaves, torch.ones_like(out), retain_graph=True)
        got = torch.autograd.grad(out.sum(), leaves)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
