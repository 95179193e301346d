"""The model's operators at the edges of what their callers may do, on the GPU."""
import numpy as np
import pytest
import torch

import operators_reference as ref
from gpu_util import binding, to_dev

pytestmark = pytest.mark.gpu


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
