"""Calls of the norms, the short convolution and the selective scan at the edges of what their documentation allows."""
import numpy as np
import pytest
import torch

import operators_reference as ref
import state_space_reference as ssr
from gpu_util import binding, to_dev
from test_gpu_state_space import SCAN_GRADS, dev, norm, real, wide

pytestmark = pytest.mark.gpu


# the longest rows that a team holds, and rows beyond the registers, of one row and of several to a share of the columns' sums
@pytest.mark.parametrize("dtype,T,D", [("f16", 3, 16384), ("f16", 3, 20001), ("bf16", 7, 16391), ("f32", 5, 8192), ("f32", 3, 8197),
                                       ("f32", 1500, 8195)])
@pytest.mark.parametrize("center", [False, True])
def test_norm_gradients_in_the_place_of_what_they_come_from(dtype, T, D, center):
    """dx in the place of dout or dsum: the weights' gradients are still those of dout."""
    print(f"norm in place T={T} D={D} {dtype} center {center}", flush=True)
    bl = binding()
    x, dy, ds = (torch.randn((1, T, D), device="cuda").to(ref.TORCH[dtype]) for _ in range(3))
    w = torch.randn(D, device="cuda")
    valid = (torch.rand((1, T), device="cuda") < 0.8).to(torch.uint8)
    valid[0, 0] = 1
    _, stats = bl.bload_layer_norm(x, w, valid=valid, center=center, training=True)
    want = bl.bload_layer_norm_backward(dy, x, stats, w, valid=valid, dsum=ds, center=center)
    for place in (0, 1):
        a, b = dy.clone(), ds.clone()
        to = ((a, b)[place], torch.empty_like(w), torch.empty_like(w))
        bl.bload_layer_norm_backward(a, x, stats, w, valid=valid, dsum=b, center=center, grads=to)
        for name, got, there in zip(("dx", "dweight", "dbias"), to, want):
            assert torch.equal(got, there), (name, ("dout", "dsum")[place])


def overflowing(T, N, dtype, each, seed=0):
    """Inputs of a scan whose states grow: where a sequence starts, its step times the rate is beyond what an exponential in 32 bits
    holds; inside a sequence it is small.  Every `each` slots a sequence starts, some after padding."""
    rng = np.random.default_rng([T, N, seed])
    B, D, G = 3, 7, 1
    reset, valid = np.zeros((B, T), np.uint8), np.ones((B, T), np.uint8)
    reset[:, ::each] = 1
    valid[1, 1::4 * each] = 0
    reset[1] *= (rng.random(T) < 0.5).astype(np.uint8) | np.r_[1, valid[1, :-1]].astype(np.uint8)
    starts = (valid == 1) & ((reset == 1) | np.concatenate([np.ones((B, 1), bool), valid[:, :-1] == 0], 1))
    t = dict(x=ref.draw(rng, (B, T, D), dtype), b=ref.draw(rng, (B, T, G, N), dtype), c=ref.draw(rng, (B, T, G, N), dtype),
             z=ref.draw(rng, (B, T, D), dtype), skip=real(rng, D), rate=1 + real(rng, D, N).abs())
    steps = np.where(starts[..., None], 100.0, 0.01) * (1 + rng.random((B, T, D)))
    t["dt"] = torch.from_numpy(steps.astype(np.float32)).to(ref.TORCH[dtype])
    return reset, valid, t, ref.draw(rng, (B, T, D), dtype), real(rng, B, D, N)


# the form for single tokens, blocks of a few slots, whole blocks and blocks that are cut
@pytest.mark.parametrize("T,N,dtype,each,train", [(1, 5, "f32", 1, False), (1, 16, "bf16", 1, False), (6, 8, "f16", 2, False), (6, 16, "f32", 3, True),
                                                  (40, 16, "f32", 1, True), (77, 24, "f32", 5, True), (300, 4, "bf16", 7, True),
                                                  (2100, 5, "f32", 3, True)])
def test_scan_a_start_drops_the_state_however_large_its_step(T, N, dtype, each, train):
    """Where a sequence starts the state is step b x, and no decay has a part in it: none that overflows either."""
    print(f"scan of large steps T={T} N={N} {dtype} each {each} train {train}", flush=True)
    bl = binding()
    reset, valid, t, dout, ds = overflowing(T, N, dtype, each)
    d = {k: dev(v) for k, v in t.items()}
    pos, args = [d[k] for k in ("x", "dt", "rate", "b", "c")], dict(skip=d["skip"], z=d["z"], softplus=False)
    flags = to_dev(reset), to_dev(valid)
    got = dict(zip(("out", "state", "saved"), bl.bload_selective_scan(*pos, *flags, **args, training=train)))
    if train:
        got.update(zip(SCAN_GRADS, bl.bload_selective_scan_backward(dev(dout), *pos, *flags, got["saved"], **args, dstate=dev(ds))))
    want = ssr.scan(*(wide(t[k]) for k in ("x", "dt", "rate", "b", "c")), reset, valid, wide(t["skip"]), wide(t["z"]), None, False, None, dtype,
                    wide(dout), wide(ds))
    for name, value in got.items():
        if name != "saved" and value is not None:
            ref.assert_close(value, *want[name], f"{name} T={T} N={N} {dtype}")


# More rows than workgroups take in one turn, and as many as make a team take several at a time, with a rest: for teams of 4, 8 (of
# single elements as well), 16, 32 and 64 lanes, of 256 and 512, and for rows beyond the registers.
@pytest.mark.parametrize("B,T,H,D,dtype", [(2, 65551, 4, 5, "f32"), (3, 43711, 4, 9, "bf16"), (1, 524401, 1, 3, "f16"), (1, 131101, 2, 33, "f16"),
                                           (3, 43711, 1, 65, "bf16"), (5, 13127, 1, 129, "bf16"), (1, 10937, 3, 257, "f16"), (2, 8219, 1, 513, "bf16"),
                                           (1, 16421, 1, 513, "f32"), (1, 16411, 1, 1025, "bf16"), (3, 1373, 1, 2049, "bf16"), (1, 4111, 1, 2049, "f32"),
                                           (1, 4109, 1, 4097, "f16"), (1, 1100, 1, 4097, "f32"), (1, 1100, 1, 8193, "bf16"), (2, 550, 1, 8197, "f32")])
def test_norm_of_many_rows(B, T, H, D, dtype):
    print(f"norm B={B} T={T} H={H} D={D} {dtype}", flush=True)
    norm(B, T, H, D, dtype, True, D % 2 == 1 and D < 1000, True, True)


@pytest.mark.parametrize("T,D,dtype", [(4099, 4097, "f32"), (4099, 8193, "f16"), (4099, 8197, "f32")])
def test_norm_of_many_long_rows_forward(T, D, dtype):
    print(f"norm T={T} D={D} {dtype}", flush=True)
    norm(1, T, 1, D, dtype, False, False, True, False)


# More shares of the runs than workgroups, so that each takes several; blocks of several runs of 16, 32, 64 and 128 slots and a rest.
# Lanes that share a wavefront's run (D of 66, 132 in 16 bits), rows of no whole number of pieces, rows below one piece.
@pytest.mark.parametrize("B,T,D,K,dtype", [(30000, 131, 1, 4, "f32"), (44000, 70, 3, 4, "f32"), (1400, 130, 66, 4, "f32"), (1400, 130, 67, 3, "f32"),
                                           (1400, 260, 66, 4, "f32"), (1400, 130, 132, 4, "bf16"), (1400, 130, 133, 4, "f16")])
def test_conv_of_many_runs(B, T, D, K, dtype):
    print(f"conv B={B} T={T} D={D} K={K} {dtype}", flush=True)
    bl = binding()
    # (as many parts of the weights' gradients as there are workgroups at most, each of which takes more than one share)
    assert bl.bload_segment_conv_backward_workspace_bytes(B, T, D, K, ref.TORCH[dtype]) == -(-1024 * D * (K + 1) * 4 // 16) * 16
    rng = np.random.default_rng([B, T, D, K])
    reset, valid, _, _ = ref.flags(rng, B, T, 30)
    reset[:, 0] &= rng.integers(0, 2, B).astype(np.uint8)
    x, dout = (ref.draw(rng, (B, T, D), dtype) for _ in range(2))
    s0, ds = (ref.draw(rng, (B, K - 1, D), dtype) for _ in range(2))
    w, b = real(rng, D, K), real(rng, D)
    args = dev(w), to_dev(reset), to_dev(valid)
    y, last = bl.bload_segment_conv(dev(x), *args, bias=dev(b), silu=True, state_in=dev(s0))
    grads = bl.bload_segment_conv_backward(dev(dout), dev(x), *args, bias=dev(b), silu=True, state_in=dev(s0), dstate=dev(ds))
    want = ssr.conv(wide(x), wide(w), wide(b), reset, valid, True, wide(s0), dtype, wide(dout), wide(ds))
    for name, got in zip(("out", "state", "dx", "dweight", "dbias", "dstate_in"), (y, last, *grads)):
        value, off = want[name]
        if name in ("dweight", "dbias"):
            # what the form allows is 200 roundings of the sum of sizes.  An addend goes through at most 2 shares of 128 slots in its lane,
            # 6 lanes, 4 wavefronts, 64 parts and 16 shares of them: 346, in twice as many.
            off = 2 * off
        ref.assert_close(got, value, off, f"{name} B={B} T={T} D={D} K={K} {dtype}")
