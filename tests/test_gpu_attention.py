"""Attention inside the sequences of packed blocks (mask, forward, backward, single queries) on the GPU against the
64-bit forms of operators_reference.py, whose bounds were derived there."""
import numpy as np
import pytest
import torch

import operators_reference as ref
from gpu_util import binding, to_dev

pytestmark = pytest.mark.gpu

NAMES = ("out", "lse", "dq", "dk", "dv")


def placed(t, how):
    """The same values in device memory, laid out in another way."""
    B, T, H, D = t.shape
    if how == "plain":
        return t.cuda()
    if how == "fused":                                       # among other heads
        big = torch.full((B, T, H + 3, D), float("nan"), dtype=t.dtype, device="cuda")
        big[:, :, 1:1 + H] = t.cuda()
        return big[:, :, 1:1 + H]
    if how == "heads_first":                                 # [B, H, T, D]
        return t.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
    raw = torch.full((B * T * H * (D + 1) + 1,), float("nan"), dtype=t.dtype, device="cuda")      # rows D + 1 apart, from element 1 on
    view = raw[1:].view(B, T, H, D + 1)[..., :D]
    view.copy_(t.cuda())
    return view


def run(B, T, Hq, Hkv, D, dtype, causal=True, pre=False, cap=0.0, bias=False, mean=40, how="plain", spoil=None, seed=0):
    """One forward and backward pass, everything checked against the reference."""
    bl = binding()
    rng = np.random.default_rng([B, T, Hq, D, seed])
    reset, valid, seq_id, n = ref.flags(rng, B, T, mean)
    prefix = rng.integers(-1, 30, n).astype(np.int32) if pre else None
    see = ref.visible(reset, valid, seq_id, causal, prefix)
    slopes = rng.random(Hq).astype(np.float32) if bias else None
    q, k, v, g = (ref.draw(rng, (B, T, h, D), dtype) for h in (Hq, Hkv, Hkv, Hq))
    scale = 1.0 / np.sqrt(D)
    want = ref.attention(ref.wide(q), ref.wide(k), ref.wide(v), see, scale, cap, slopes, dtype, ref.wide(g))
    dead = np.zeros((B, T), bool)
    if spoil:
        dead = spoil(valid, seq_id, (q, k, v, g))
    dq, dk, dv, dg = (placed(t, how) for t in (q, k, v, g))
    mask = bl.bload_segment_mask(to_dev(reset), to_dev(valid), causal=causal, prefix=to_dev(prefix) if pre else None, seq_id=to_dev(seq_id))
    kw = dict(cap=cap, slopes=to_dev(slopes) if bias else None)
    out, saved = bl.bload_segment_attention(dq, dk, dv, mask, training=True, **kw)
    grads = [placed(torch.full_like(t, float("nan")), how) for t in (q, k, v)]
    bl.bload_segment_attention_backward(dg, dq, dk, dv, out, saved, mask, grads=grads, **kw)
    torch.cuda.synchronize()
    got = dict(zip(NAMES, (out, saved.lse, *grads)))
    live = ~dead
    for name in NAMES:
        value, bound = want[name]
        x = ref.wide(got[name])
        if name == "lse":
            x, value, bound = (np.moveaxis(y, 1, 2) for y in (x, value, bound))
        ref.assert_close(x[live], value[live], bound[live], f"{name} B={B} T={T} Hq={Hq} Hkv={Hkv} D={D} {dtype} causal {causal} {how}")
        if name != "lse":
            assert not x[valid == 0].any(), f"{name}: padding is not zero"
    return bl, (dq, dk, dv, dg, mask, kw), got


# lengths on both sides of every tile (32, 64, 128), heads on both sides of every padded size (32, 64, 96, 128)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,T,Hq,Hkv,D", [(1, 1, 1, 1, 1), (2, 2, 2, 1, 8), (3, 31, 4, 4, 16), (2, 33, 4, 2, 31), (2, 64, 6, 2, 32),
                                          (1, 65, 3, 1, 33), (2, 127, 2, 2, 37), (1, 128, 4, 1, 64), (2, 129, 2, 1, 65), (1, 200, 2, 2, 80),
                                          (1, 257, 2, 1, 96), (1, 190, 3, 3, 97), (1, 300, 4, 2, 128), (5, 40, 2, 2, 127)])
def test_sizes(B, T, Hq, Hkv, D, dtype):
    for causal in (True, False):
        print(f"attention B={B} T={T} Hq={Hq} Hkv={Hkv} D={D} {dtype} causal {causal}", flush=True)
        run(B, T, Hq, Hkv, D, dtype, causal)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D", [20, 64, 90, 128])
@pytest.mark.parametrize("causal,pre,cap,bias", [(True, True, 0.0, False), (True, False, 5.0, False), (False, False, 0.0, True),
                                                 (True, True, 2.0, True), (False, False, 30.0, True)])
def test_masks_caps_and_slopes(causal, pre, cap, bias, D, dtype):
    print(f"attention D={D} {dtype} causal {causal} prefix {pre} cap {cap} slopes {bias}", flush=True)
    run(2, 170, 4, 2, D, dtype, causal, pre, cap, bias)


@pytest.mark.parametrize("mean", [1.2, 8, 1000])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_lengths_of_sequences(mean, dtype):
    """Blocks of single frames, of many short sequences and of one that fills the block."""
    run(2, 333, 2, 1, 48, dtype, True, mean=mean)
    run(2, 333, 2, 1, 48, dtype, False, mean=mean)


@pytest.mark.parametrize("how", ["fused", "heads_first", "odd"])
@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 37), ("f32", 24), ("f32", 5)])
def test_strides(how, dtype, D):
    run(2, 150, 4, 2, D, dtype, how=how)


def poison_padding(valid, seq_id, tensors):
    for t in tensors:
        t[torch.from_numpy(valid == 0)] = float("nan")
    tensors[1][torch.from_numpy(valid == 0)] = float("inf")
    return np.zeros(valid.shape, bool)


def poison_a_sequence(valid, seq_id, tensors):
    """One sequence in each block is lost: the others must not notice."""
    dead = np.zeros(valid.shape, bool)
    for b in range(valid.shape[0]):
        ids = seq_id[b][seq_id[b] >= 0]
        dead[b] = seq_id[b] == ids[len(ids) // 2]
    for t, x in zip(tensors, (float("inf"), float("nan"), float("-inf"), float("nan"))):
        t[torch.from_numpy(dead)] = x
    return dead


@pytest.mark.parametrize("spoil", [poison_padding, poison_a_sequence])
@pytest.mark.parametrize("dtype,D,cap", [("f16", 64, 0.0), ("bf16", 100, 5.0), ("f32", 30, 0.0)])
def test_what_is_hidden_has_no_part(spoil, dtype, D, cap):
    run(2, 150, 4, 2, D, dtype, True, cap=cap, spoil=spoil, mean=20)
    run(2, 150, 4, 2, D, dtype, False, cap=cap, spoil=spoil, mean=20)


def test_later_frames_have_no_part():
    """Causally, a frame that is not a number is seen only by those behind it; its own query spoils the keys it sees."""
    bl = binding()
    T, H, D, at = 140, 2, 64, 70
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((1, T, H, D), generator=g).half().cuda() for _ in range(3))
    reset, valid = torch.zeros((1, T), dtype=torch.uint8, device="cuda"), torch.ones((1, T), dtype=torch.uint8, device="cuda")
    mask = bl.bload_segment_mask(reset, valid)
    clean = bl.bload_segment_attention(q, k, v, mask)
    v2 = v.clone()
    v2[:, at] = float("nan")
    dirty = bl.bload_segment_attention(q, k, v2, mask)
    assert torch.isnan(dirty[:, at:]).all()
    # (the rows of the spoiled tile are computed by other means: equal to a step of the type)
    assert (dirty[:, :at].float() - clean[:, :at].float()).abs().max() <= 2.0 ** -9


def test_row_of_infinitely_low_scores_is_not_a_number():
    bl = binding()
    q = torch.ones((1, 4, 1, 8), device="cuda")
    k = torch.full((1, 4, 1, 8), float("-inf"), device="cuda")
    k[0, 3] = 1.0
    v = torch.ones_like(q)
    flags = torch.zeros((1, 4), dtype=torch.uint8, device="cuda")
    out = bl.bload_segment_attention(q, k, v, bl.bload_segment_mask(flags, flags + 1))
    assert torch.isnan(out[0, :3]).all() and torch.equal(out[0, 3], v[0, 3])      # softmax over -inf alone has no value


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("B,T,mean", [(1, 1, 1), (3, 7, 2), (2, 1023, 50), (2, 1024, 3000), (3, 1025, 4000), (2, 5000, 9000), (1, 20000, 3000)])
def test_mask(B, T, mean, causal):
    bl = binding()
    rng = np.random.default_rng([B, T])
    reset, valid, seq_id, n = ref.flags(rng, B, T, mean, 0.02)
    prefix = rng.integers(-2, 2 * mean + 2, max(1, n)).astype(np.int32)
    want = np.zeros((B, T, 4), np.int32)
    for b in range(B):
        for f, e in ref.segments(reset[b], valid[b]):
            t = np.arange(f, e)
            h = f + min(max(0, int(prefix[seq_id[b, f]])), e - f)
            want[b, f:e] = np.stack([0 * t + f, np.maximum(t + 1, h) if causal else 0 * t + e, np.where(causal & (t >= h), t, f), 0 * t + e], 1)
    got = bl.bload_segment_mask(to_dev(reset), to_dev(valid), causal=bool(causal), prefix=to_dev(prefix), seq_id=to_dev(seq_id))
    assert np.array_equal(got.cpu().numpy(), want)


def test_same_inputs_same_bits_on_any_stream_and_in_a_graph():
    bl, (q, k, v, g, mask, kw), first = run(3, 260, 4, 2, 64, "bf16", True, cap=10.0)
    want = [first[n].clone() for n in NAMES]
    ws = torch.empty(bl.bload_segment_attention_backward_workspace_bytes(3, 260, 4), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        out, saved = bl.bload_segment_attention(q, k, v, mask, training=True, **kw)
        return (out, saved.lse, *bl.bload_segment_attention_backward(g, q, k, v, out, saved, mask, workspace=ws, **kw))
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for replay in range(3):
        q.copy_(torch.randn_like(q))
        eager = [t.clone() for t in step()]
        for t in held:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), f"replay {replay}"


def test_gradients_are_differences_of_the_forward_pass():
    """float32: the loss along a direction, two forward passes 2 e apart.  The forward pass is off by some 1e-6 of each
    of its n terms, which random signs add up to sqrt(n), so the quotient by 1e-6 sqrt(n) / e; the third
    derivative's share is e^2 times the gradient's size."""
    bl = binding()
    g = torch.Generator(device="cuda").manual_seed(2)
    B, T, H, D, e = 2, 60, 2, 16, 1e-2
    new = lambda: torch.randn((B, T, H, D), device="cuda", generator=g)
    q, k, v, w = new(), new(), new(), new()
    flags = torch.zeros((B, T), dtype=torch.uint8, device="cuda")
    flags[:, 25] = 1
    mask = bl.bload_segment_mask(flags, torch.ones_like(flags))
    out, saved = bl.bload_segment_attention(q, k, v, mask, cap=4.0, training=True)
    grads = bl.bload_segment_attention_backward(w, q, k, v, out, saved, mask, cap=4.0)
    for i in range(3):
        d = new()

        def loss(step):
            x = [t + step * d if i == j else t for j, t in enumerate((q, k, v))]
            return float((bl.bload_segment_attention(*x, mask, cap=4.0).double() * w.double()).sum())
        rise = (loss(e) - loss(-e)) / (2 * e)
        want = float((grads[i].double() * d.double()).sum())
        size = float((grads[i].double() * d.double()).abs().sum())
        assert abs(rise - want) <= 1e-6 * (B * T * H * D) ** 0.5 / e + 10 * e * e * size


# ---------------------------------------------------------------- single queries


def decode(n, B, T, Hq, Hkv, D, dtype, lengths, cap=0.0, bias=False, how="plain", seed=0):
    bl = binding()
    rng = np.random.default_rng([n, T, Hq, D, seed])
    L = np.asarray(lengths)[np.arange(n) % len(lengths)].astype(np.int32)
    block = rng.integers(0, B, n).astype(np.int32)
    offset = np.array([rng.integers(0, T - x + 1) for x in L], np.int32)
    slopes = rng.random(Hq).astype(np.float32) / 8 if bias else None
    q, k, v = ref.draw(rng, (n, 1, Hq, D), dtype), ref.draw(rng, (B, T, Hkv, D), dtype), ref.draw(rng, (B, T, Hkv, D), dtype)
    dk, dv = placed(k, how), placed(v, how)
    got = bl.bload_segment_attention_decode(q[:, 0].cuda(), dk, dv, to_dev(block), to_dev(offset), to_dev(L), cap=cap,
                                            slopes=to_dev(slopes) if bias else None)
    K, V, Q = ref.wide(k), ref.wide(v), ref.wide(q)
    for i in range(n):
        if L[i] == 0:
            assert not got[i].any()
            continue
        at = slice(offset[i], offset[i] + L[i])
        qq = np.zeros((1, L[i], Hq, D))
        qq[0, -1] = Q[i, 0]
        see = np.zeros((1, L[i], L[i]), bool)
        see[0, -1] = True
        value, bound = ref.attention(qq, K[block[i]:block[i] + 1, at], V[block[i]:block[i] + 1, at], see, D ** -0.5, cap, slopes, dtype)["out"]
        ref.assert_close(got[i], value[0, -1], bound[0, -1], f"decode sequence {i} of {L[i]} frames, T={T} Hq={Hq} Hkv={Hkv} D={D} {dtype}")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n,B,T,Hq,Hkv,D,lengths", [(1, 1, 1, 1, 1, 1, [1]), (3, 2, 40, 4, 2, 64, [0, 1, 40]), (5, 2, 300, 8, 1, 37, [31, 32, 33, 300, 2]),
                                                    (4, 3, 1500, 6, 6, 128, [1500, 129, 127, 700]), (2, 1, 700, 40, 1, 80, [700, 65]),
                                                    (6, 2, 2100, 64, 2, 16, [2100, 3, 1025])])
def test_decode(n, B, T, Hq, Hkv, D, lengths, dtype):
    print(f"decode n={n} T={T} Hq={Hq} Hkv={Hkv} D={D} {dtype}", flush=True)
    decode(n, B, T, Hq, Hkv, D, dtype, lengths)
    decode(n, B, T, Hq, Hkv, D, dtype, lengths, cap=3.0, bias=True, seed=1)


@pytest.mark.parametrize("how", ["fused", "heads_first", "odd"])
def test_decode_strides(how):
    decode(3, 2, 200, 4, 2, 48, "f16", [200, 77, 1], how=how)
    decode(3, 2, 200, 4, 2, 33, "bf16", [200, 77, 1], how=how)


def test_decode_answers_zero_for_what_is_not_there():
    bl = binding()
    q, k = torch.ones((6, 2, 16), device="cuda"), torch.ones((2, 10, 1, 16), device="cuda")
    got = bl.bload_segment_attention_decode(q, k, k, *(to_dev(np.array(x, np.int32)) for x in
                                                       ([-1, 2, 0, 1, 0, 1], [0, 0, -1, 6, 0, 6], [3, 3, 3, 5, -4, 4])))
    assert not got[:5].any() and torch.equal(got[5], torch.ones_like(got[5]))


def test_decode_offsets_beyond_32_bits():
    bl = binding()
    B, T, H, D = 5, 1 << 17, 32, 128                        # 2.7e9 elements
    kv = torch.zeros((B, T, H, D), dtype=torch.float16, device="cuda")
    kv[B - 1, T - 3:] = 1.0
    q = torch.ones((2, H, D), dtype=torch.float16, device="cuda")
    tables = [to_dev(np.array(x, np.int32)) for x in ([B - 1, B - 1], [T - 3, T - 6], [3, 3])]
    got = bl.bload_segment_attention_decode(q, kv, kv, *tables)
    assert torch.equal(got[0], torch.ones_like(got[0])) and not got[1].any()


def test_attention_offsets_beyond_32_bits():
    """Blocks whose elements lie beyond 2^31, reached through strides: the last two blocks of a tall tensor."""
    bl = binding()
    B, T, H, D = 2, 96, 2, 64
    stride = (1 << 31) + 128
    raw = torch.zeros(stride + T * H * D, dtype=torch.float16, device="cuda")
    view = raw.as_strided((B, T, H, D), (stride, H * D, D, 1))
    x = torch.randn((B, T, H, D), device="cuda").half()
    view.copy_(x)
    flags = torch.zeros((B, T), dtype=torch.uint8, device="cuda")
    mask = bl.bload_segment_mask(flags, flags + 1)
    out, saved = bl.bload_segment_attention(view, view, view, mask, training=True)
    grads = bl.bload_segment_attention_backward(view, view, view, view, out, saved, mask)
    want, kept = bl.bload_segment_attention(x, x, x, mask, training=True)
    wants = bl.bload_segment_attention_backward(x, x, x, x, want, kept, mask)
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(grads, wants))
