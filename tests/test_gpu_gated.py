"""The gated recurrence and rotary positions on the GPU against the 64-bit forms of operators_reference.py."""
import numpy as np
import pytest
import torch

import operators_reference as ref
from gpu_util import Guarded, binding, to_dev

pytestmark = pytest.mark.gpu


def gated(B, T, D, dtype, state, mean, seed=0, gates="sigmoid"):
    bl = binding()
    rng = np.random.default_rng([B, T, D, seed])
    reset, valid, _, _ = ref.flags(rng, B, T, mean)
    if state:
        reset[:, 0] &= rng.integers(0, 2, B).astype(np.uint8)
    a = rng.standard_normal((B, T, D)).astype(np.float32)
    gate = torch.from_numpy(1 / (1 + np.exp(-2 - 1.5 * a)) if gates == "sigmoid" else np.tanh(2 * a)).to(ref.TORCH[dtype])
    x, w = ref.draw(rng, (B, T, D), dtype), ref.draw(rng, (B, T, D), dtype)
    h0 = torch.from_numpy(rng.standard_normal((B, D)).astype(np.float32)) if state else None
    ws = torch.from_numpy(rng.standard_normal((B, D)).astype(np.float32)) if state else None
    dev = lambda t: None if t is None else t.cuda()
    d_reset, d_valid = to_dev(reset), to_dev(valid)
    h, last = bl.bload_gated_scan(dev(gate), dev(x), d_reset, d_valid, h0=dev(h0))
    grads = bl.bload_gated_scan_backward(dev(w), dev(gate), h, d_reset, d_valid, h0=dev(h0), dstate=dev(ws))
    torch.cuda.synchronize()
    wide = lambda t: None if t is None else ref.wide(t)
    want = ref.gated(wide(gate), wide(x), reset, valid, wide(h0), dtype, wide(w), wide(ws))
    what = f"B={B} T={T} D={D} {dtype} state {state} mean {mean}"
    for name, got in zip(("h", "state", "dgate", "dx", "dh0"), (h, last, *grads)):
        ref.assert_close(got, *want[name], f"{name} {what}")
        if name in ("h", "dgate", "dx"):
            assert not ref.wide(got)[valid == 0].any()


# rows of less than 16 bytes, of odd numbers of elements, of several slices; blocks below and beyond the short form,
# of a step's length and one slot more, cut into chunks and whole
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,T,D", [(1, 1, 1), (5, 1, 2048), (3, 8, 37), (2, 9, 1), (4, 33, 7), (2, 64, 64), (3, 65, 129), (2, 257, 80),
                                   (1, 2049, 3), (2, 1000, 260), (1, 5000, 1), (1, 4097, 33), (600, 40, 16), (520, 70, 300)])
def test_gated(B, T, D, dtype):
    for state, mean in ((False, 10), (True, 300)):
        print(f"gated B={B} T={T} D={D} {dtype} state {state}", flush=True)
        gated(B, T, D, dtype, state, mean)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_gated_signs_and_long_memories(dtype):
    gated(2, 700, 40, dtype, True, 5000, gates="tanh")
    gated(2, 3000, 24, dtype, True, 100000, 1)


@pytest.mark.parametrize("B,T,D", [(2, 6, 24), (2, 300, 24), (600, 50, 40)])
def test_gated_what_is_cut_off_has_no_part(B, T, D):
    """A lost sequence and spoiled padding: the sequences around them come out as if they were not there."""
    bl = binding()
    rng = np.random.default_rng(T)
    reset, valid, seq_id, n = ref.flags(rng, B, T, 4)
    lost = (valid == 0) | (seq_id % 3 == 1)
    gate, x, w = (torch.rand((B, T, D)).cuda() for _ in range(3))
    d_reset, d_valid, d_lost = to_dev(reset), to_dev(valid), torch.from_numpy(lost).cuda()

    def both(gate, x, w):
        h, _ = bl.bload_gated_scan(gate, x, d_reset, d_valid)
        return (h, *bl.bload_gated_scan_backward(w, gate, h, d_reset, d_valid)[:2])
    clean = both(gate, x, w)
    for t, bad in ((gate, float("inf")), (x, float("nan")), (w, float("-inf"))):
        t[d_lost] = bad
    for a, b in zip(both(gate, x, w), clean):
        assert torch.equal(a[~d_lost], b[~d_lost])
        assert not a[d_valid == 0].any()


def test_gated_writes_inside_its_outputs():
    bl = binding()
    B, T, D = 3, 130, 37
    rng = np.random.default_rng(1)
    reset, valid, _, _ = ref.flags(rng, B, T, 20)
    gate, x = torch.rand((B, T, D)).half().cuda(), torch.randn((B, T, D)).half().cuda()
    g = [Guarded(B * T * D * 2) for _ in range(3)] + [Guarded(B * D * 4) for _ in range(2)]
    h, dgate, dx = (t.view(torch.float16, (B, T, D)) for t in g[:3])
    state, dh0 = (t.view(torch.float32, (B, D)) for t in g[3:])
    bl.bload_gated_scan(gate, x, to_dev(reset), to_dev(valid), out=h, state=state)
    bl.bload_gated_scan_backward(x, gate, h, to_dev(reset), to_dev(valid), grads=(dgate, dx, dh0))
    torch.cuda.synchronize()
    assert all(t.intact() for t in g)
    assert not dh0.any()                                     # no state went in


def test_gated_stream_of_single_frames_equals_the_block():
    """One frame at a time with the state handed on, the state's buffer in place, and blocks that continue one another."""
    bl = binding()
    B, T, D = 7, 24, 40
    gate, x = torch.rand((B, T, D), device="cuda"), torch.randn((B, T, D), device="cuda")
    reset, valid = torch.zeros((B, T), dtype=torch.uint8, device="cuda"), torch.ones((B, T), dtype=torch.uint8, device="cuda")
    reset[2, 9] = 1
    state = torch.randn((B, D), device="cuda")
    whole, last = bl.bload_gated_scan(gate, x, reset, valid, h0=state)
    one = state.clone()
    cut = lambda t, a, b: t[:, a:b].contiguous()
    for t in range(T):
        h, _ = bl.bload_gated_scan(cut(gate, t, t + 1), cut(x, t, t + 1), cut(reset, t, t + 1), cut(valid, t, t + 1), h0=one, state=one)
        assert torch.allclose(h[:, 0], whole[:, t], rtol=1e-5, atol=1e-5)
    assert torch.allclose(one, last, rtol=1e-5, atol=1e-5)
    h1, s1 = bl.bload_gated_scan(cut(gate, 0, 10), cut(x, 0, 10), cut(reset, 0, 10), cut(valid, 0, 10), h0=state)
    h2, s2 = bl.bload_gated_scan(cut(gate, 10, T), cut(x, 10, T), cut(reset, 10, T), cut(valid, 10, T), h0=s1)
    assert torch.allclose(torch.cat([h1, h2], 1), whole, rtol=1e-5, atol=1e-5) and torch.allclose(s2, last, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,T,H,D,rot", [(1, 1, 1, 2, 2), (2, 9, 3, 7, 4), (3, 40, 5, 64, 64), (2, 33, 2, 80, 20), (2, 50, 40, 128, 128),
                                         (1, 17, 3, 74, 18), (2, 5, 9, 37, 36), (1, 300, 70, 16, 10)])
def test_rotary(B, T, H, D, rot, layout, dtype):
    bl = binding()
    rng = np.random.default_rng([T, D, rot])
    x = ref.draw(rng, (B, T, H, D), dtype)
    pos = rng.integers(0, 5000, (B, T)).astype(np.int32)
    pos.flat[rng.integers(0, B * T, max(1, B * T // 6))] = -1
    pos[0, 0] = (1 << 31) - 1 if T > 1 else 12345
    freq = bl.bload_rotary_frequencies(rot, 1000.0, 4.0, 500)
    big = torch.full((B, T, H + 2, D), float("nan"), dtype=x.dtype, device="cuda")
    big[:, :, 1:1 + H] = x.cuda()
    # an angle of 2^31 radians in 64 bits is off by 2^-22 radians; sine and cosine, two products and a sum round in 32
    for inverse, scale in ((False, 1.0), (True, 0.75)):
        want, size = ref.rotary(ref.wide(x), pos, freq.double().numpy(), layout, scale, inverse)
        bound = (2.0 ** -21 * (pos[..., None, None] > 1 << 20) + 8 * ref.U32) * size + ref.half_step(dtype) * np.abs(want) + ref.tiny(dtype)
        got = bl.bload_rotary(big[:, :, 1:1 + H], to_dev(pos), freq.cuda(), layout, scale, inverse)
        ref.assert_close(got, want, bound, f"rotary {layout} B={B} T={T} H={H} D={D} rot={rot} {dtype}")
        same = big[:, :, 1:1 + H].clone()
        assert torch.equal(bl.bload_rotary(same, to_dev(pos), freq.cuda(), layout, scale, inverse, out=same), got)      # in place
    assert torch.isnan(big[:, :, 0]).all() and torch.isnan(big[:, :, -1]).all()


def test_gated_and_rotary_replay_in_a_graph():
    bl = binding()
    B, T, D = 2, 500, 64
    rng = np.random.default_rng(0)
    reset, valid, _, _ = ref.flags(rng, B, T, 50)
    reset, valid = to_dev(reset), to_dev(valid)
    gate, x = torch.rand((B, T, D), device="cuda"), torch.randn((B, T, D), device="cuda")
    pos, freq = torch.arange(B * T, dtype=torch.int32, device="cuda").view(B, T), bl.bload_rotary_frequencies(32).cuda()
    ws = torch.empty(bl.bload_gated_scan_workspace_bytes(B, T, D, torch.float32), dtype=torch.uint8, device="cuda")

    def step():
        h, s = bl.bload_gated_scan(gate, x, reset, valid, workspace=ws)
        g = bl.bload_gated_scan_backward(x, gate, h, reset, valid, workspace=ws)
        return [h, s, *g, bl.bload_rotary(x.view(B, T, 2, 32), pos, freq)]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for replay in range(3):
        x.copy_(torch.randn_like(x))
        eager = [t.clone() for t in step()]
        for t in held:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), f"replay {replay}"
