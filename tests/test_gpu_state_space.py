"""Norms, the short convolution and the selective scan on the GPU against the 64-bit forms of state_space_reference.py."""
import numpy as np
import pytest
import torch

import operators_reference as ref
import state_space_reference as ssr
from gpu_util import Guarded, binding, to_dev

pytestmark = pytest.mark.gpu

wide = lambda t: None if t is None else ref.wide(t)
dev = lambda t: None if t is None else t.cuda()
real = lambda rng, *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32))


def inside(t, dtype=None):
    """The tensor as a part of a larger one, between NaNs: slots further apart, blocks too, the start at no multiple of 16 bytes."""
    shape = list(t.shape)
    shape[0], shape[1], shape[-1] = shape[0], shape[1] + 1, shape[-1] + 3
    big = torch.full(shape, float("nan"), dtype=t.dtype, device="cuda")
    part = big[:, :-1, ..., 1:-2]
    part.copy_(t)
    return part


# ---------------------------------------------------------------- norms


def norm(B, T, H, D, dtype, center, residual, masked, train, strided=False, eps=1e-5, mean=0.25, weights=True, seed=0):
    bl = binding()
    rng = np.random.default_rng([B, T, H, D, seed])
    shape = (B, T, H, D) if H > 1 else (B, T, D)
    x = (real(rng, *shape) * 1.5 + mean).to(ref.TORCH[dtype])
    res, dout, dsum = (ref.draw(rng, shape, dtype) for _ in range(3))
    w, b = (real(rng, D) * 0.2 + 1, real(rng, D)) if weights else (None, None)
    valid = (rng.random((B, T)) < 0.8).astype(np.uint8) if masked else None
    live = np.ones(B * T, bool) if valid is None else valid.reshape(-1) != 0
    put = inside if strided else dev
    if valid is not None and not strided:
        x[torch.from_numpy(valid) == 0] = float("nan")       # what padding holds has no part
    got = bl.bload_layer_norm(put(x), dev(w), dev(b) if center else None, residual=put(res) if residual else None,
                              valid=None if valid is None else to_dev(valid), eps=eps, center=center, training=train)
    got = list(got) if isinstance(got, tuple) else [got]
    s = (x.float() + res.float()).to(x.dtype) if residual else x
    flat = lambda t: np.nan_to_num(ref.wide(t).reshape(-1, D))
    want = ssr.norm(flat(s), wide(w), wide(b) if center else None, live.repeat(H), eps, center, dtype, flat(dout), flat(dsum) if residual else None)
    what = f"norm {shape} {dtype} center {center} residual {residual} masked {masked} strided {strided}"
    ref.assert_close(ref.wide(got[0]).reshape(-1, D), *want["out"], what)
    if residual:
        assert np.array_equal(ref.wide(got[1]).reshape(-1, D)[live.repeat(H)], flat(s)[live.repeat(H)]), what
        assert not ref.wide(got[1]).reshape(-1, D)[~live.repeat(H)].any(), what
    if not train:
        return
    stats = ref.wide(got[-1]).reshape(-1, 2)
    ref.assert_close(stats[:, 1:], *want["r"], "1 / deviation " + what)
    dx, dw, db = bl.bload_layer_norm_backward(put(dout), got[1] if residual else put(x), got[-1], dev(w),
                                              valid=None if valid is None else to_dev(valid), dsum=put(dsum) if residual else None, center=center)
    ref.assert_close(ref.wide(dx).reshape(-1, D), *want["dx"], "dx " + what)
    ref.assert_close(dw, *want["dweight"], "dweight " + what)
    ref.assert_close(db, *want["dbias"], "dbias " + what)


# rows on both sides of every number of lanes and pieces, below one piece, of no whole number of pieces, and beyond the registers
NORM_SHAPES = [(1, 1, 1, 1), (2, 3, 1, 2), (3, 5, 2, 7), (2, 9, 3, 8), (2, 7, 5, 33), (3, 11, 2, 64), (2, 17, 6, 128), (1, 40, 3, 129), (2, 33, 1, 255),
               (2, 15, 1, 512), (2, 9, 1, 515), (1, 13, 1, 1024), (1, 11, 1, 1025), (1, 9, 1, 2048), (1, 7, 1, 2051), (2, 5, 1, 4096), (1, 5, 1, 4099),
               (1, 4, 1, 8192), (1, 3, 1, 8197), (1, 3, 1, 16384), (1, 3, 1, 16391), (40, 32, 1, 64), (3, 700, 4, 24)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,T,H,D", NORM_SHAPES)
def test_norm(B, T, H, D, dtype):
    print(f"norm B={B} T={T} H={H} D={D} {dtype}", flush=True)
    norm(B, T, H, D, dtype, True, False, True, True)
    norm(B, T, H, D, dtype, True, True, True, True, seed=1)
    norm(B, T, H, D, dtype, False, False, False, True, strided=True)
    norm(B, T, H, D, dtype, False, True, False, False, weights=False, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_rows_far_from_zero(dtype):
    """Means much larger than deviations: the variance is that of the differences."""
    for D in (96, 1000, 3000, 20000):
        norm(2, 9, 1, D, dtype, True, False, True, True, mean=100.0)


def test_norm_of_equal_elements_and_of_what_is_not_finite():
    bl = binding()
    x = torch.full((1, 4, 300), 2.5, device="cuda")
    x[0, 1, 7], x[0, 2, 9] = float("nan"), float("inf")
    bias = torch.arange(300, device="cuda", dtype=torch.float32)
    y = bl.bload_layer_norm(x, None, bias, eps=1e-5)
    assert torch.equal(y[0, 0], bias) and torch.equal(y[0, 3], bias)         # no deviation: the bias is left
    assert torch.isnan(y[0, 1]).all() and torch.isnan(y[0, 2]).all()


def test_norm_in_place_and_inside_its_outputs():
    bl = binding()
    for B, T, D in ((3, 50, 37), (2, 9, 2051), (1, 3, 20001)):
        x, res, dy = (torch.randn((B, T, D), device="cuda").half() for _ in range(3))
        valid = (torch.rand((B, T), device="cuda") < 0.8).to(torch.uint8)
        y, total, stats = bl.bload_layer_norm(x, residual=res, valid=valid, training=True)
        xx, rr = x.clone(), res.clone()
        got = bl.bload_layer_norm(xx, residual=rr, valid=valid, out=xx, total=rr)
        assert got[0] is xx and torch.equal(xx, y) and torch.equal(rr, total)
        dx, dw, db = bl.bload_layer_norm_backward(dy, total, stats, valid=valid, dsum=res)
        for place in (0, 1):
            a, b = dy.clone(), res.clone()
            bl.bload_layer_norm_backward(a, total, stats, valid=valid, dsum=b, grads=((a, b)[place], None, None))
            assert torch.equal((a, b)[place], dx)
        g = [Guarded(B * T * D * 2) for _ in range(3)] + [Guarded(D * 4) for _ in range(2)]
        half = [t.view(torch.float16, (B, T, D)) for t in g[:3]]
        bl.bload_layer_norm(x, residual=res, valid=valid, out=half[0], total=half[1])
        bl.bload_layer_norm_backward(dy, total, stats, valid=valid, dsum=res, grads=(half[2], *(t.view(torch.float32, (D,)) for t in g[3:])))
        torch.cuda.synchronize()
        assert all(t.intact() for t in g) and torch.equal(half[2], dx)


# ---------------------------------------------------------------- short convolution


def conv(B, T, D, K, dtype, silu, state, mean, strided=False, bias=True, seed=0):
    bl = binding()
    rng = np.random.default_rng([B, T, D, K, seed])
    reset, valid, _, _ = ref.flags(rng, B, T, mean)
    if state:
        reset[:, 0] &= rng.integers(0, 2, B).astype(np.uint8)
    x, dout = (ref.draw(rng, (B, T, D), dtype) for _ in range(2))
    s0, ds = (ref.draw(rng, (B, K - 1, D), dtype) if state else None for _ in range(2))
    w, b = real(rng, D, K), real(rng, D) if bias else None
    put = inside if strided else dev
    d_reset, d_valid = to_dev(reset), to_dev(valid)
    y, last = bl.bload_segment_conv(put(x), dev(w), d_reset, d_valid, bias=dev(b), silu=silu, state_in=dev(s0))
    grads = bl.bload_segment_conv_backward(put(dout), put(x), dev(w), d_reset, d_valid, bias=dev(b), silu=silu, state_in=dev(s0), dstate=dev(ds))
    torch.cuda.synchronize()
    want = ssr.conv(wide(x), wide(w), wide(b), reset, valid, silu, wide(s0), dtype, wide(dout), wide(ds))
    what = f"conv B={B} T={T} D={D} K={K} {dtype} silu {silu} state {state} mean {mean} strided {strided}"
    for name, got in zip(("out", "state", "dx", "dweight", "dbias", "dstate_in"), (y, last, *grads)):
        ref.assert_close(got, *want[name], f"{name} {what}")


# blocks below, at and beyond a run and a step; rows below one piece, of no whole number of pieces, of several slices
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,T,D,K", [(1, 1, 1, 1), (5, 1, 200, 4), (3, 2, 37, 4), (2, 5, 9, 8), (4, 16, 7, 3), (2, 17, 64, 4), (3, 33, 129, 2),
                                     (2, 67, 3, 5), (2, 130, 80, 4), (1, 300, 520, 4), (2, 257, 33, 6), (1, 65, 1030, 4), (300, 20, 8, 7),
                                     (2, 1500, 24, 4)])
def test_conv(B, T, D, K, dtype):
    print(f"conv B={B} T={T} D={D} K={K} {dtype}", flush=True)
    conv(B, T, D, K, dtype, True, False, 10)
    conv(B, T, D, K, dtype, True, True, 3, strided=True)
    conv(B, T, D, K, dtype, False, True, 100, bias=False, seed=1)


def test_conv_many_runs_to_a_workgroup():
    conv(2100, 65, 520, 4, "f16", True, False, 30)


@pytest.mark.parametrize("K", [2, 4, 8])
def test_conv_state_in_place_and_a_stream_of_single_frames(K):
    bl = binding()
    B, T, D = 7, 24, 41
    x = torch.randn((B, T, D), device="cuda")
    w, b = torch.randn((D, K), device="cuda"), torch.randn(D, device="cuda")
    reset, valid = torch.zeros((B, T), dtype=torch.uint8, device="cuda"), torch.ones((B, T), dtype=torch.uint8, device="cuda")
    reset[2, 9] = 1
    s0 = torch.randn((B, K - 1, D), device="cuda")
    whole, last = bl.bload_segment_conv(x, w, reset, valid, bias=b, silu=True, state_in=s0)
    for step in (1, 3, 8):
        one, at = s0.clone(), 0
        while at < T:
            cut = lambda t: t[:, at:at + step]
            y, same = bl.bload_segment_conv(cut(x), w, cut(reset).contiguous(), cut(valid).contiguous(), bias=b, silu=True, state_in=one, state=one)
            assert same is one and torch.equal(y, cut(whole))
            at += step
        assert torch.equal(one, last)


# ---------------------------------------------------------------- selective scan


def scan_inputs(rng, B, T, D, N, G, dtype, z, softplus, state):
    t = dict(x=ref.draw(rng, (B, T, D), dtype), b=ref.draw(rng, (B, T, G, N), dtype), c=ref.draw(rng, (B, T, G, N), dtype))
    t["rate"] = -(1 + torch.arange(N)) * torch.exp(0.2 * real(rng, D, N))
    t["z"] = ref.draw(rng, (B, T, D), dtype) if z else None
    t["skip"] = real(rng, D)
    steps = torch.exp(torch.from_numpy(rng.uniform(np.log(1e-3), np.log(0.3), D).astype(np.float32)))
    if softplus:
        t["dt"], t["dt_bias"] = ref.draw(rng, (B, T, D), dtype), torch.log(torch.expm1(steps))
    else:
        t["dt"], t["dt_bias"] = (steps * (1 + real(rng, B, T, D).abs())).to(ref.TORCH[dtype]), None
    t["h0"] = real(rng, B, D, N) if state else None
    return t


SCAN_GRADS = ("dx", "ddt", "drate", "db", "dc", "dskip", "dz", "ddt_bias", "dh0")


def scan(B, T, D, N, G, dtype, z, softplus, state, mean, strided=False, seed=0):
    bl = binding()
    rng = np.random.default_rng([B, T, D, N, G, seed])
    reset, valid, _, _ = ref.flags(rng, B, T, mean)
    if state:
        reset[:, 0] &= rng.integers(0, 2, B).astype(np.uint8)
    t = scan_inputs(rng, B, T, D, N, G, dtype, z, softplus, state)
    dout, ds = ref.draw(rng, (B, T, D), dtype), real(rng, B, D, N) if state else None
    put = inside if strided else dev
    d = {k: put(v) if k in ("x", "dt", "z", "b", "c") and v is not None else dev(v) for k, v in t.items()}
    pos = [d.pop(k) for k in ("x", "dt", "rate", "b", "c")]
    flags = to_dev(reset), to_dev(valid)
    y, last, saved = bl.bload_selective_scan(*pos, *flags, **d, softplus=softplus, training=True)
    plain, last2 = bl.bload_selective_scan(*pos, *flags, **d, softplus=softplus)
    grads = bl.bload_selective_scan_backward(put(dout), *pos, *flags, saved, **d, softplus=softplus, dstate=dev(ds))
    torch.cuda.synchronize()
    want = ssr.scan(*(wide(t[k]) for k in ("x", "dt", "rate", "b", "c")), reset, valid, wide(t["skip"]), wide(t["z"]), wide(t["dt_bias"]),
                    softplus, wide(t["h0"]), dtype, wide(dout), wide(ds))
    what = f"scan B={B} T={T} D={D} N={N} G={G} {dtype} z {z} softplus {softplus} state {state} mean {mean} strided {strided}"
    for name, got in (("out", y), ("state", last), ("out", plain), ("state", last2), *zip(SCAN_GRADS, grads)):
        assert (got is None) == (name == "dz" and not z or name == "ddt_bias" and not softplus or name == "dh0" and not state)
        if got is not None:
            ref.assert_close(got, *want[name], f"{name} {what}")


# blocks of one slot, below and beyond the short form, at the edges of a tile, of several chunks; channels below and beyond a
# workgroup's, in groups of no whole number of them; every number of states a lane may hold
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,T,D,N,G", [(1, 1, 1, 1, 1), (5, 1, 200, 16, 1), (3, 8, 37, 5, 1), (2, 9, 2, 1, 2), (4, 15, 64, 16, 1), (2, 16, 70, 8, 2),
                                       (3, 17, 65, 4, 1), (2, 33, 130, 16, 1), (2, 100, 24, 24, 3), (1, 130, 20, 33, 1), (2, 65, 12, 64, 1),
                                       (1, 300, 10, 2, 1), (1, 1000, 6, 16, 1), (2, 2100, 3, 7, 1), (90, 40, 66, 16, 1)])
def test_scan(B, T, D, N, G, dtype):
    print(f"scan B={B} T={T} D={D} N={N} G={G} {dtype}", flush=True)
    scan(B, T, D, N, G, dtype, True, True, False, 10)
    scan(B, T, D, N, G, dtype, True, True, True, 300, strided=True, seed=1)
    scan(B, T, D, N, G, dtype, False, False, True, 30, seed=2)


def test_scan_several_blocks_to_a_workgroup():
    scan(4500, 9, 5, 4, 1, "f32", True, True, True, 20)


@pytest.mark.parametrize("B,T,D,N", [(2, 6, 24, 8), (2, 300, 24, 16), (500, 40, 20, 16)])
def test_scan_and_conv_what_is_cut_off_has_no_part(B, T, D, N):
    """A lost sequence and spoiled padding: the sequences around them come out as if they were not there."""
    bl = binding()
    rng = np.random.default_rng(T)
    reset, valid, seq_id, _ = ref.flags(rng, B, T, 4)
    lost = torch.from_numpy((valid == 0) | (seq_id % 3 == 1)).cuda()
    d_reset, d_valid = to_dev(reset), to_dev(valid)
    t = {k: dev(v) for k, v in scan_inputs(rng, B, T, D, N, 1, "f32", True, True, False).items()}
    w, dout = torch.randn((D, 4), device="cuda"), torch.randn((B, T, D), device="cuda")

    def all_of():
        args = dict(skip=t["skip"], z=t["z"], dt_bias=t["dt_bias"])
        pos = [t[k] for k in ("x", "dt", "rate", "b", "c")]
        y, _, saved = bl.bload_selective_scan(*pos, d_reset, d_valid, **args, training=True)
        plain = bl.bload_selective_scan(*pos, d_reset, d_valid, **args)[0]
        g = bl.bload_selective_scan_backward(dout, *pos, d_reset, d_valid, saved, **args)
        v, _ = bl.bload_segment_conv(t["x"], w, d_reset, d_valid, silu=True)
        dv = bl.bload_segment_conv_backward(dout, t["x"], w, d_reset, d_valid, silu=True)[0]
        n = bl.bload_layer_norm(t["x"], valid=d_valid)
        return [y, plain, g[0], g[1], g[3].flatten(2), g[4].flatten(2), g[6], v, dv, n]
    clean = all_of()
    for name, bad in (("x", float("nan")), ("dt", float("inf")), ("z", float("nan")), ("b", float("inf")), ("c", float("-inf")), ("dout", float("inf"))):
        spoilt = dout if name == "dout" else t[name]
        spoilt[lost] = bad
        for i, (got, want) in enumerate(zip(all_of(), clean)):
            assert torch.equal(got[~lost], want[~lost]), (name, i)
            assert not got[d_valid == 0].any(), (name, i)


def test_scan_state_in_place_and_a_stream_of_single_frames():
    bl = binding()
    rng = np.random.default_rng(5)
    for D, N in ((41, 16), (70, 5), (9, 64)):
        B, T = 6, 24
        t = {k: dev(v) for k, v in scan_inputs(rng, B, T, D, N, 1, "f32", True, True, True).items()}
        reset, valid = torch.zeros((B, T), dtype=torch.uint8, device="cuda"), torch.ones((B, T), dtype=torch.uint8, device="cuda")
        reset[2, 9] = 1
        args = dict(skip=t["skip"], dt_bias=t["dt_bias"])
        whole, last = bl.bload_selective_scan(t["x"], t["dt"], t["rate"], t["b"], t["c"], reset, valid, z=t["z"], h0=t["h0"], **args)
        for step in (1, 3, 8):
            one, at = t["h0"].clone(), 0
            while at < T:
                cut = lambda v: v[:, at:at + step]
                x, dt, b, c, z = (cut(t[k]) for k in ("x", "dt", "b", "c", "z"))
                flags = cut(reset).contiguous(), cut(valid).contiguous()
                apart, other = bl.bload_selective_scan(x, dt, t["rate"], b, c, *flags, z=z, h0=one, **args)
                y, same = bl.bload_selective_scan(x, dt, t["rate"], b, c, *flags, z=z, h0=one, state=one, **args)
                assert same is one and torch.equal(y, apart) and torch.equal(one, other)
                # the same products in another order of additions over N states
                assert torch.allclose(y, cut(whole), rtol=1e-4, atol=1e-4)
                at += step
            assert torch.allclose(one, last, rtol=1e-5, atol=1e-5)


def test_scan_and_conv_write_inside_their_outputs():
    bl = binding()
    rng = np.random.default_rng(1)
    for B, T, D, N in ((3, 130, 37, 5), (2, 7, 70, 16), (1, 40, 130, 33)):
        reset, valid, _, _ = ref.flags(rng, B, T, 20)
        t = {k: dev(v) for k, v in scan_inputs(rng, B, T, D, N, 1, "f16", True, True, True).items()}
        flags = to_dev(reset), to_dev(valid)
        dout = torch.randn((B, T, D), device="cuda").half()
        pos, args = [t[k] for k in ("x", "dt", "rate", "b", "c")], dict(skip=t["skip"], z=t["z"], dt_bias=t["dt_bias"], h0=t["h0"])
        y, state, saved = bl.bload_selective_scan(*pos, *flags, **args, training=True)
        want = bl.bload_selective_scan_backward(dout, *pos, *flags, saved, **args)
        slots = Guarded(y.numel() * 2), Guarded(state.numel() * 4)
        bl.bload_selective_scan(*pos, *flags, **args, out=slots[0].view(y.dtype, y.shape), state=slots[1].view(state.dtype, state.shape))
        g = [Guarded(v.numel() * v.element_size()) for v in want]
        views = [a.view(v.dtype, v.shape) for a, v in zip(g, want)]
        bl.bload_selective_scan_backward(dout, *pos, *flags, saved, **args, grads=views)
        w, s0 = torch.randn((D, 4), device="cuda"), torch.randn((B, 3, D), device="cuda").half()
        cy, cs = bl.bload_segment_conv(t["x"], w, *flags, silu=True, state_in=s0)
        cg = bl.bload_segment_conv_backward(dout, t["x"], w, *flags, silu=True, state_in=s0)
        gc = [Guarded(v.numel() * v.element_size()) for v in (cy, cs, *cg)]
        cv = [a.view(v.dtype, v.shape) for a, v in zip(gc, (cy, cs, *cg))]
        bl.bload_segment_conv(t["x"], w, *flags, silu=True, state_in=s0, out=cv[0], state=cv[1])
        bl.bload_segment_conv_backward(dout, t["x"], w, *flags, silu=True, state_in=s0, grads=cv[2:])
        torch.cuda.synchronize()
        assert all(a.intact() for a in (*slots, *g, *gc))
        # (twice the same call: the same bits)
        assert all(torch.equal(a, b) for a, b in zip(views, want)) and all(torch.equal(a, b) for a, b in zip(cv, (cy, cs, *cg)))


def layer_pass(bl, t, flags, dout, w, work):
    """Norm, convolution, scan and their gradients, as a layer runs them; every workspace brought along."""
    B, T, D = t["x"].shape
    n, stats = bl.bload_layer_norm(t["x"], valid=flags[1], training=True)
    v, vs = bl.bload_segment_conv(n, w, *flags, silu=True)
    pos, args = [v, *(t[k] for k in ("dt", "rate", "b", "c"))], dict(skip=t["skip"], z=t["z"], dt_bias=t["dt_bias"])
    y, last, saved = bl.bload_selective_scan(*pos, *flags, **args, training=True, workspace=work[0])
    g = bl.bload_selective_scan_backward(dout, *pos, *flags, saved, **args, workspace=work[1])
    gv = bl.bload_segment_conv_backward(g[0], n, w, *flags, silu=True, workspace=work[2])
    gn = bl.bload_layer_norm_backward(gv[0], t["x"], stats, valid=flags[1], workspace=work[3])
    return [n, v, vs, y, last, *(x for x in g if x is not None), *gv, *gn]


def test_layer_of_all_three_replays_in_a_graph_and_on_another_stream():
    bl = binding()
    B, T, D, N = 2, 500, 72, 16
    rng = np.random.default_rng(0)
    reset, valid, _, _ = ref.flags(rng, B, T, 50)
    flags = to_dev(reset), to_dev(valid)
    t = {k: dev(v) for k, v in scan_inputs(rng, B, T, D, N, 1, "bf16", True, True, False).items()}
    dout, w = torch.randn((B, T, D), device="cuda").bfloat16(), torch.randn((D, 4), device="cuda")
    sizes = (bl.bload_selective_scan_workspace_bytes(B, T, D, N), bl.bload_selective_scan_backward_workspace_bytes(B, T, D, N),
             bl.bload_segment_conv_backward_workspace_bytes(B, T, D, 4, torch.bfloat16),
             bl.bload_layer_norm_backward_workspace_bytes(B, T, 1, D, torch.bfloat16))
    assert min(sizes) > 0
    work = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    step = lambda: layer_pass(bl, t, flags, dout, w, work)
    first = [x.clone() for x in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for replay in range(3):
        t["x"].copy_(torch.randn_like(t["x"]))
        dout.copy_(torch.randn_like(dout))
        eager = [x.clone() for x in step()]
        for x in held:
            x.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), f"replay {replay}"


def test_nothing_to_do():
    """No blocks: gradients of weights are zeros."""
    bl = binding()
    z3 = lambda *s: torch.empty(s, device="cuda")
    flags = torch.empty((0, 5), dtype=torch.uint8, device="cuda")
    dx, dw, db = bl.bload_layer_norm_backward(z3(0, 5, 8), z3(0, 5, 8), z3(0, 5, 2))
    assert not dw.any() and not db.any()
    got = bl.bload_segment_conv_backward(z3(0, 5, 8), z3(0, 5, 8), torch.ones((8, 4), device="cuda"), flags, flags)
    assert not got[1].any() and not got[2].any()
    rate, skip = torch.ones((8, 3), device="cuda"), torch.ones(8, device="cuda")
    args = z3(0, 5, 8), z3(0, 5, 8), rate, z3(0, 5, 1, 3), z3(0, 5, 1, 3), flags, flags
    y, s, saved = bl.bload_selective_scan(*args, skip=skip, training=True)
    got = bl.bload_selective_scan_backward(z3(0, 5, 8), *args, saved, skip=skip)
    assert not got[2].any() and not got[5].any()


def test_offsets_beyond_32_bits():
    """Blocks whose elements lie beyond 2^31, reached through strides."""
    bl = binding()
    B, T, D, N = 2, 50, 64, 16
    stride = (1 << 31) + 128
    raw = torch.zeros(stride + 8 * T * D, dtype=torch.float16, device="cuda")
    rng = np.random.default_rng(8)
    t = {k: dev(v) for k, v in scan_inputs(rng, B, T, D, N, 1, "f16", True, True, False).items()}
    far = dict(t)
    at = 0
    for k in ("x", "dt", "z", "b", "c"):
        shape = t[k].shape
        size = shape[1:].numel()
        far[k] = raw.as_strided(shape, (stride, size // T, *((N, 1) if len(shape) == 4 else (1,))), at)
        far[k].copy_(t[k])
        at += size
    dout = torch.randn((B, T, D), device="cuda").half()
    far_out = raw.as_strided((B, T, D), (stride, D, 1), at)
    far_out.copy_(dout)
    reset, valid, _, _ = ref.flags(rng, B, T, 20)
    flags, w = (to_dev(reset), to_dev(valid)), torch.randn((D, 4), device="cuda")

    def all_of(t, dout):
        pos, args = [t[k] for k in ("x", "dt", "rate", "b", "c")], dict(skip=t["skip"], z=t["z"], dt_bias=t["dt_bias"])
        y, s, saved = bl.bload_selective_scan(*pos, *flags, **args, training=True)
        n = bl.bload_layer_norm(t["x"], training=True)
        return [y, s, *bl.bload_selective_scan_backward(dout, *pos, *flags, saved, **args)[:8], *bl.bload_segment_conv(t["x"], w, *flags, silu=True),
                *bl.bload_segment_conv_backward(dout, t["x"], w, *flags, silu=True), *n, *bl.bload_layer_norm_backward(dout, t["x"], n[1])]
    assert all(torch.equal(a, b) for a, b in zip(all_of(t, dout), all_of(far, far_out)))


def test_long_memories_and_large_steps():
    """Steps that keep everything, steps after which nothing is left, and rates of 0: no decay at all."""
    bl = binding()
    rng = np.random.default_rng(9)
    B, T, D, N = 2, 1500, 5, 4
    t = scan_inputs(rng, B, T, D, N, 1, "f32", False, False, False)
    t["dt"] = torch.from_numpy(np.exp(rng.uniform(np.log(1e-6), np.log(1e3), (B, T, D))).astype(np.float32))
    t["rate"][0] = 0
    t["rate"][1] *= 1e-4
    one = np.ones((B, T), np.uint8)
    got = bl.bload_selective_scan(*(dev(t[k]) for k in ("x", "dt", "rate", "b", "c")), to_dev(0 * one), to_dev(one), softplus=False)
    want = ssr.scan(*(wide(t[k]) for k in ("x", "dt", "rate", "b", "c")), 0 * one, one, None, None, None, False, None, "f32")
    ref.assert_close(got[0], *want["out"], "long memories")
    ref.assert_close(got[1], *want["state"], "long memories, state")
