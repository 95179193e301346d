"""What the attention, rotary and gated-recurrence entry points refuse, and their workspace queries: answered on the
host, before anything is launched (no GPU)."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000
OK, EINVAL, ELENGTH, EWORKSPACE, EALIGN, EOVERFLOW = range(6)
F16, F32, I32, BF16 = 1, 2, 3, 4


@pytest.fixture(scope="module")
def bl():
    if not os.path.exists(os.path.join(ROOT, "paper_2310_10879_amd", "libbload.so")):
        from paper_2310_10879_amd import build
        build.build(verbose=False)
    from paper_2310_10879_amd import bload
    return bload


def heads(bl, p=P):
    return bl.Heads(p, 1024, 128, 64)


def test_mask(bl):
    f = bl._lib.bload_segment_mask

    def call(reset=P, valid=P, seq_id=P, B=4, T=100, causal=1, prefix=None, n=0, out=P):
        return f(reset, valid, seq_id, B, T, causal, prefix, n, out, None)
    assert call(B=-1) == call(T=0) == call(n=-1) == call(causal=2) == EINVAL
    assert call(reset=None) == call(valid=None) == call(out=None) == EINVAL
    assert call(prefix=P, seq_id=None, n=3) == EINVAL
    assert call(out=P + 8) == call(prefix=P + 2) == call(seq_id=P + 1) == EALIGN
    assert call(T=(1 << 30) + 1) == call(B=1 << 40) == call(n=(1 << 27) + 1) == EOVERFLOW
    assert call(B=0, reset=None, valid=None, out=None) == OK


def attention_args(bl, backward, **kw):
    a = dict(q=heads(bl), k=heads(bl), v=heads(bl), mask=P, B=4, T=100, Hq=4, Hkv=2, D=64, dtype=F16, scale=0.1, cap=0.0, slopes=None,
             out=heads(bl), lse=P, rest=None, dout=heads(bl), dq=heads(bl), dk=heads(bl), dv=heads(bl), ws=P, room=1 << 30)
    a.update(kw)
    sizes = [a[n] for n in ("B", "T", "Hq", "Hkv", "D", "dtype", "scale", "cap", "slopes")]
    if backward:
        return bl._lib.bload_segment_attention_backward(a["dout"], a["q"], a["k"], a["v"], a["out"], a["lse"], a["rest"], a["mask"], *sizes,
                                                        a["dq"], a["dk"], a["dv"], a["ws"], a["room"], None)
    return bl._lib.bload_segment_attention(a["q"], a["k"], a["v"], a["mask"], *sizes, a["out"], a["lse"], a["rest"], None)


@pytest.mark.parametrize("backward", [False, True])
def test_attention(bl, backward):
    call = lambda **kw: attention_args(bl, backward, **kw)
    for bad in (dict(B=-1), dict(T=0), dict(Hq=0), dict(Hkv=0), dict(Hq=5), dict(D=0), dict(D=129), dict(dtype=0), dict(dtype=I32),
                dict(dtype=5), dict(dtype=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")),
                dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(mask=None), dict(q=None), dict(k=None), dict(v=None),
                dict(out=None), dict(q=heads(bl, None)), dict(out=heads(bl, 0))):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(mask=P + 4), dict(slopes=P + 2), dict(q=heads(bl, P + 1)), dict(v=heads(bl, P + 2), dtype=F32), dict(lse=P + 2),
                dict(rest=heads(bl, P + 1))):
        assert call(**bad) == EALIGN, bad
    assert call(T=(1 << 30) + 1) == call(B=1 << 40) == call(B=1 << 24, T=1 << 14, Hq=64) == EOVERFLOW
    assert call(B=0, q=None, k=None, v=None, out=None, mask=None) == OK
    if backward:
        for name in ("dout", "dq", "dk", "dv"):
            assert call(**{name: None}) == EINVAL
            assert call(**{name: heads(bl, P + 1)}) == EALIGN
        assert call(lse=None) == call(ws=None) == EINVAL
        assert call(ws=P + 8) == EALIGN
        assert call(room=4 * 4 * 100 * 4 - 1) == EWORKSPACE


def test_decode(bl):
    f = bl._lib.bload_segment_attention_decode

    def call(q=heads(bl), k=heads(bl), v=heads(bl), block=P, offset=P, length=P, n=3, B=4, T=100, Hq=4, Hkv=2, D=64, dtype=F16, scale=0.1,
             cap=0.0, slopes=None, out=heads(bl), ws=P, room=1 << 40):
        return f(q, k, v, block, offset, length, n, B, T, Hq, Hkv, D, dtype, scale, cap, slopes, out, ws, room, None)
    for bad in (dict(n=-1), dict(B=-1), dict(T=0), dict(Hq=3), dict(D=129), dict(dtype=I32), dict(scale=0.0), dict(cap=-1.0), dict(q=None),
                dict(out=None), dict(k=None), dict(v=heads(bl, None)), dict(block=None), dict(offset=None), dict(length=None)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(block=P + 1), dict(offset=P + 2), dict(length=P + 3), dict(q=heads(bl, P + 1)), dict(slopes=P + 1)):
        assert call(**bad) == EALIGN, bad
    assert call(n=(1 << 27) + 1) == call(B=1 << 40) == call(n=1 << 27, Hq=64, Hkv=64) == EOVERFLOW
    assert call(n=0, q=None, k=None, v=None, out=None, block=None) == OK
    need = bl.bload_segment_attention_decode_workspace_bytes(3, 30000, 4, 2, 64)
    assert need > 0
    assert call(T=30000, room=need - 1) == EWORKSPACE and call(T=30000, ws=None) == EINVAL and call(T=30000, ws=P + 4) == EALIGN
    assert bl.bload_segment_attention_decode_workspace_bytes(100000, 100, 4, 2, 64) == 0
    assert bl.bload_segment_attention_decode_workspace_bytes(3, 30000, 4, 3, 64) == 0


def test_gated(bl):
    fwd, bwd = bl._lib.bload_gated_scan, bl._lib.bload_gated_scan_backward

    def forward(gate=P, x=P, reset=P, valid=P, B=4, T=100, D=64, dtype=F16, h0=None, out=P, state=None, ws=P, room=1 << 40):
        return fwd(gate, x, reset, valid, B, T, D, dtype, h0, out, state, ws, room, None)

    def backward(dout=P, gate=P, h=P, reset=P, valid=P, B=4, T=100, D=64, dtype=F16, h0=None, dstate=None, dgate=P, dx=P, dh0=None, ws=P,
                 room=1 << 40):
        return bwd(dout, gate, h, reset, valid, B, T, D, dtype, h0, dstate, dgate, dx, dh0, ws, room, None)
    for f in (forward, backward):
        for bad in (dict(B=-1), dict(T=0), dict(D=0), dict(dtype=0), dict(dtype=I32), dict(dtype=9), dict(gate=None), dict(reset=None),
                    dict(valid=None)):
            assert f(**bad) == EINVAL, bad
        assert f(T=(1 << 30) + 1) == f(D=(1 << 30) + 1) == f(B=1 << 40) == EOVERFLOW
        assert f(gate=P + 1) == f(h0=P + 2) == f(gate=P + 2, dtype=F32) == EALIGN
        assert f(T=5000, room=bl.bload_gated_scan_workspace_bytes(4, 5000, 64, torch.float16) // 64) == EWORKSPACE
        assert f(T=5000, ws=None) == EINVAL and f(T=5000, ws=P + 8) == EALIGN
        assert f(B=0, gate=None) == OK
    assert forward(x=None) == forward(out=None) == EINVAL and forward(state=P + 1) == forward(out=P + 1) == EALIGN
    assert backward(dout=None) == backward(h=None) == backward(dgate=None) == backward(dx=None) == EINVAL
    assert backward(dh0=P + 2) == backward(dstate=P + 1) == backward(dx=P + 1) == EALIGN
    assert bl.bload_gated_scan_workspace_bytes(4096, 1, 2048, torch.bfloat16) == 0
    assert bl.bload_gated_scan_workspace_bytes(0, 100, 64, torch.float32) == 0


def test_rotary(bl):
    f = bl._lib.bload_rotary

    def call(x=heads(bl), pos=P, B=4, T=100, H=4, D=64, dtype=F16, freq=P, rot=64, layout=0, scale=1.0, inverse=0, out=heads(bl)):
        return f(x, pos, B, T, H, D, dtype, freq, rot, layout, scale, inverse, out, None)
    for bad in (dict(B=-1), dict(T=0), dict(H=0), dict(D=0), dict(dtype=0), dict(dtype=I32), dict(rot=0), dict(rot=3), dict(rot=66),
                dict(layout=2), dict(scale=float("nan")), dict(inverse=2), dict(x=None), dict(out=None), dict(pos=None), dict(freq=None)):
        assert call(**bad) == EINVAL, bad
    assert call(pos=P + 2) == call(freq=P + 1) == call(x=heads(bl, P + 1)) == call(out=heads(bl, P + 2), dtype=F32) == EALIGN
    assert call(B=1 << 40) == call(B=1 << 26, T=1 << 13, D=4096, rot=2) == EOVERFLOW
    assert call(B=0, x=None) == OK


def test_rotary_frequencies(bl):
    f = bl.bload_rotary_frequencies
    plain = f(16, 500.0)
    want = 500.0 ** (-torch.arange(0, 16, 2, dtype=torch.float64) / 16)
    assert torch.equal(plain, want.float())
    assert torch.equal(f(16, 500.0, factor=4.0), (want / 4).float())
    turns = 100 * want / (2 * torch.pi)
    keep = ((turns - 1.0) / 7.0).clamp(0, 1)
    assert 0 < int(((keep > 0) & (keep < 1)).sum()) < 8
    assert torch.allclose(f(16, 500.0, 4.0, 100, 1.0, 8.0).double(), want * (keep + (1 - keep) / 4), rtol=1e-7, atol=0)
    for bad in ((3, 10.0), (0, 10.0), (4, 0.0), (4, float("inf")), (4, 10.0, 0.0), (4, 10.0, 1.0, -1), (4, 10.0, 1.0, 5, 8.0, 8.0)):
        with pytest.raises(bl.BloadError):
            f(*bad)


def test_old_entry_points_still_refuse_the_new_type(bl):
    p, z = ctypes.c_void_p(P), ctypes.c_void_p(None)
    assert bl._lib.bload_segment_reduce(p, p, p, p, 5, 8, 8, BF16, 0, 3, p, z, 0, z) == EINVAL
    assert bl._lib.bload_segment_scan(p, p, p, 5, 8, 8, BF16, 0.5, p, z, 0, z) == EINVAL
    assert bl._lib.bload_segment_reduce_workspace_bytes(5, 8, 8, BF16) == bl._lib.bload_segment_scan_workspace_bytes(5, 8, 8, BF16) == 0


def test_binding_checks_its_tensors(bl):
    cpu = torch.zeros(2, 8, 4, 16)
    with pytest.raises(ValueError):
        bl.bload_segment_attention(cpu, cpu, cpu, torch.zeros(2, 8, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        bl.bload_segment_attention(cpu.double(), cpu, cpu, torch.zeros(2, 8, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        bl.bload_rotary(cpu, torch.zeros(2, 8, dtype=torch.int32), torch.zeros(4))
    with pytest.raises(ValueError):
        bl.bload_gated_scan(cpu[:, :, 0], cpu[:, :, 0], torch.zeros(2, 8, dtype=torch.uint8), torch.zeros(2, 8, dtype=torch.uint8))
