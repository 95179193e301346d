"""What the norm, the short convolution and the selective scan refuse, and their workspace queries: answered on the host, before
anything is launched (no GPU)."""
import pytest
import torch

from test_operators_refuse import EALIGN, EINVAL, EOVERFLOW, EWORKSPACE, F16, F32, I32, OK, P, bl, heads  # noqa: F401

BIG = 1 << 40


def test_norm(bl):
    fwd, bwd = bl._lib.bload_layer_norm, bl._lib.bload_layer_norm_backward

    def forward(x=heads(bl), res=None, valid=P, B=4, T=100, H=2, D=64, dtype=F16, center=1, eps=1e-5, w=P, b=P, out=heads(bl), total=None, stats=P):
        return fwd(x, res, valid, B, T, H, D, dtype, center, eps, w, b, out, total, stats, None)

    def backward(dout=heads(bl), x=heads(bl), stats=P, valid=P, B=4, T=100, H=2, D=64, dtype=F16, center=1, w=P, dsum=None, dx=heads(bl), dw=P, db=P,
                 ws=P, room=BIG):
        return bwd(dout, x, stats, valid, B, T, H, D, dtype, center, w, dsum, dx, dw, db, ws, room, None)
    for f in (forward, backward):
        for bad in (dict(B=-1), dict(T=0), dict(H=0), dict(D=0), dict(dtype=0), dict(dtype=I32), dict(center=2), dict(center=-1), dict(x=None),
                    dict(x=heads(bl, 0))):
            assert f(**bad) == EINVAL, bad
        assert f(T=(1 << 30) + 1) == f(D=(1 << 21) + 1) == f(B=1 << 40) == f(B=1 << 21, T=1 << 9, H=2) == EOVERFLOW
        assert f(x=heads(bl, P + 1)) == f(x=heads(bl, P + 2), dtype=F32) == f(w=P + 2) == f(stats=P + 4) == EALIGN
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(out=None)):
        assert forward(**bad) == EINVAL, bad
    assert forward(B=0, x=None, out=None) == OK
    assert forward(res=heads(bl, 0)) == forward(total=heads(bl, 0)) == EINVAL and forward(res=heads(bl, P + 1)) == forward(b=P + 1) == EALIGN
    for bad in (dict(dout=None), dict(dx=None), dict(stats=None), dict(ws=None), dict(dsum=heads(bl, 0))):
        assert backward(**bad) == EINVAL, bad
    need = bl.bload_layer_norm_backward_workspace_bytes(4, 100, 2, 64, torch.float16)
    assert need > 0 and need % 16 == 0
    assert backward(room=need - 16) == EWORKSPACE and backward(ws=P + 8) == backward(dw=P + 1) == backward(db=P + 2) == EALIGN
    assert backward(B=0, x=None, dw=None, db=None, ws=None) == OK
    assert bl.bload_layer_norm_backward_workspace_bytes(0, 100, 2, 64, torch.float16) == 0
    assert bl.bload_layer_norm_backward_workspace_bytes(4, 100, 0, 64, torch.float16) == 0


def test_conv(bl):
    fwd, bwd = bl._lib.bload_segment_conv, bl._lib.bload_segment_conv_backward

    def forward(x=heads(bl), w=P, b=P, reset=P, valid=P, B=4, T=100, D=64, K=4, dtype=F16, silu=1, s0=None, out=heads(bl), s1=None):
        return fwd(x, w, b, reset, valid, B, T, D, K, dtype, silu, s0, out, s1, None)

    def backward(dout=heads(bl), x=heads(bl), w=P, b=P, reset=P, valid=P, B=4, T=100, D=64, K=4, dtype=F16, silu=1, s0=None, d1=None, dx=heads(bl),
                 dw=P, db=P, d0=None, ws=P, room=BIG):
        return bwd(dout, x, w, b, reset, valid, B, T, D, K, dtype, silu, s0, d1, dx, dw, db, d0, ws, room, None)
    for f in (forward, backward):
        for bad in (dict(B=-1), dict(T=0), dict(D=0), dict(K=0), dict(K=9), dict(dtype=0), dict(dtype=I32), dict(silu=2), dict(silu=-1), dict(x=None),
                    dict(x=heads(bl, 0)), dict(w=None), dict(reset=None), dict(valid=None)):
            assert f(**bad) == EINVAL, bad
        assert f(T=(1 << 30) + 1) == f(D=(1 << 26) + 1) == f(B=1 << 40) == EOVERFLOW
        assert f(x=heads(bl, P + 1)) == f(w=P + 2) == f(b=P + 1) == f(s0=P + 1) == f(s0=P + 2, dtype=F32) == EALIGN
    assert forward(out=None) == EINVAL and forward(s1=P + 1) == EALIGN and forward(B=0, x=None) == OK
    assert forward(B=1 << 24, T=16, D=2048) == forward(B=1 << 30, T=1, D=4096) == EOVERFLOW
    size = 4 * 3 * 64 * 2
    for a, b, t in ((BIG, BIG, 9), (BIG, BIG + size - 2, 1), (BIG + 2, BIG, 8), (BIG, BIG, 100)):
        assert forward(s0=a, s1=b, T=t) == EINVAL
        assert backward(d1=a, d0=b, T=t) == backward(s0=a, d0=b, T=t) == EINVAL
    assert backward(d1=BIG, d0=BIG, T=1) == EINVAL
    for bad in (dict(dout=None), dict(dx=None), dict(ws=None)):
        assert backward(**bad) == EINVAL, bad
    need = bl.bload_segment_conv_backward_workspace_bytes(4, 100, 64, 4, torch.float16)
    assert need > 0 and backward(room=need - 16) == EWORKSPACE
    assert backward(ws=P + 8) == backward(dw=P + 1) == backward(db=P + 2) == backward(d1=P + 1) == backward(d0=P + 1) == EALIGN
    assert backward(B=0, x=None, dw=None, db=None, ws=None) == OK
    assert bl.bload_segment_conv_backward_workspace_bytes(0, 100, 64, 4, torch.float16) == 0
    assert bl.bload_segment_conv_backward_workspace_bytes(4, 100, 64, 9, torch.float16) == 0


def test_scan(bl):
    lib = bl._lib

    def args(**kw):
        a = dict(x=heads(bl), dt=heads(bl), z=heads(bl), b=heads(bl), c=heads(bl), rate=P, skip=P, bias=P, reset=P, valid=P, h0=None, B=4, T=100, D=64,
                 N=16, G=2, dtype=F16, softplus=1)
        a.update({k: v for k, v in kw.items() if k in a})
        return bl.Selective(*a.values())

    def forward(out=heads(bl), state=None, saved=P, ws=P, room=BIG, **kw):
        return lib.bload_selective_scan(args(**kw), out, state, saved, ws, room, None)

    def backward(dout=heads(bl), saved=P, ds=None, dx=heads(bl), ddt=heads(bl), drate=P, db=heads(bl), dc=heads(bl), dskip=P, dz=heads(bl), dbias=P,
                 dh0=None, ws=P, room=BIG, **kw):
        return lib.bload_selective_scan_backward(args(**kw), dout, saved, ds, dx, ddt, drate, db, dc, dskip, dz, dbias, dh0, ws, room, None)
    none = heads(bl, 0)
    for f in (forward, backward):
        for bad in (dict(B=-1), dict(T=0), dict(D=0), dict(N=0), dict(N=65), dict(G=0), dict(G=3), dict(dtype=0), dict(dtype=I32), dict(softplus=2),
                    dict(x=none), dict(dt=none), dict(b=none), dict(c=none), dict(rate=None), dict(reset=None), dict(valid=None)):
            assert f(**bad) == EINVAL, bad
        assert f(T=(1 << 30) + 1) == f(D=(1 << 24) + 2) == f(B=1 << 40) == f(B=1 << 30, T=1, D=64) == EOVERFLOW
        assert f(B=1 << 9, T=1 << 30, D=1 << 24, N=4) == EOVERFLOW             # sizes of workspaces beyond 64 bits
        assert f(x=heads(bl, P + 1)) == f(z=heads(bl, P + 2), dtype=F32) == f(rate=P + 2) == f(skip=P + 1) == f(bias=P + 2) == f(h0=P + 2) == EALIGN
    assert lib.bload_selective_scan(None, heads(bl), None, None, None, 0, None) == EINVAL
    assert forward(out=None) == forward(out=none) == EINVAL and forward(state=P + 2) == forward(saved=P + 2) == EALIGN
    assert forward(B=0, x=none) == OK
    size = 4 * 4 * 64 * 16
    for a, b, t in ((BIG, BIG, 9), (BIG, BIG + size - 4, 1), (BIG + 4, BIG, 8), (BIG, BIG, 100)):
        assert forward(h0=a, state=b, T=t) == EINVAL
        assert backward(ds=a, dh0=b, T=t) == backward(h0=a, dh0=b, T=t) == EINVAL
    assert backward(ds=BIG, dh0=BIG, T=1) == EINVAL
    need = bl.bload_selective_scan_workspace_bytes(4, 5000, 64, 16, 2)
    assert need > 0 and forward(T=5000, room=need - 16) == EWORKSPACE and forward(T=5000, ws=None) == EINVAL and forward(T=5000, ws=P + 8) == EALIGN
    assert bl.bload_selective_scan_workspace_bytes(4096, 1, 2048, 16) == 0 and bl.bload_selective_scan_workspace_bytes(4, 5000, 64, 16, 3) == 0
    assert bl.bload_selective_scan_saved_bytes(2, 33, 10, 5) == 2 * 3 * 10 * 5 * 4
    for bad in (dict(dout=None), dict(saved=None), dict(dx=None), dict(ddt=none), dict(db=None), dict(dc=none), dict(dz=None), dict(ws=None)):
        assert backward(**bad) == EINVAL, bad
    need = bl.bload_selective_scan_backward_workspace_bytes(4, 100, 64, 16, 2)
    assert need > 0 and backward(room=need - 16) == EWORKSPACE
    for bad in (dict(ws=P + 8), dict(drate=P + 1), dict(dskip=P + 2), dict(dbias=P + 1), dict(ds=P + 2), dict(dh0=P + 1), dict(saved=P + 2)):
        assert backward(**bad) == EALIGN, bad
    assert backward(B=0, drate=None, dskip=None, dbias=None, ws=None) == OK
    assert bl.bload_selective_scan_backward_workspace_bytes(0, 100, 64, 16) == 0


def test_binding_checks_its_tensors(bl):
    cpu, flags = torch.zeros(2, 8, 16), torch.zeros(2, 8, dtype=torch.uint8)
    with pytest.raises(ValueError):
        bl.bload_layer_norm(cpu)
    with pytest.raises(ValueError):
        bl.bload_layer_norm(cpu.double())
    with pytest.raises(ValueError, match="expected \\[B, T, D\\]"):
        bl.bload_layer_norm(torch.zeros(8, 16))
    with pytest.raises(ValueError, match="groups, states"):
        bl.bload_selective_scan(cpu, cpu, torch.zeros(16, 4), torch.zeros(2, 8, 4), torch.zeros(2, 8, 4), flags, flags)
    with pytest.raises(ValueError, match="sum with a residual"):
        bl.bload_layer_norm(cpu, total=cpu)
    with pytest.raises(ValueError):
        bl.bload_segment_conv(cpu, torch.zeros(16, 4), flags, flags)
    with pytest.raises(ValueError):
        bl.bload_selective_scan(cpu, cpu, torch.zeros(16, 4), torch.zeros(2, 8, 1, 4), torch.zeros(2, 8, 1, 4), flags, flags)
