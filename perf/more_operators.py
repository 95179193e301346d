"""Performance cases of the operators of a state space layer on packed blocks.

The packer leaves blocks ``[B, T, ...]`` of whole sequences with a start table.  A case is a dict of
plain values; ``kind`` says which operator one pass goes through:

    norm   layer norm (``center``) or root mean square norm of every slot or every head, with the sum of a
           residual stream where ``residual`` is set, and the backward pass where ``train`` is set
    conv   the short causal convolution inside the sequences of the blocks, forward and, with ``train``,
           backward; ``state`` hands in and out the last inputs, which with T = 1 is the form for single frames
    scan   the selective state space scan with the blocks' resets, in the same forms

``lengths`` names the mix of sequence lengths (see ``draw_lengths``).  The lengths belong to the case
and the seed draws the order of the blocks and the payload, so that every seed fills tensors of the
same shape.  With ``own`` false a pass is plain torch in 32 bits, with ``own`` true it makes the calls of
``paper_2310_10879_amd.bload``.  ``exact`` gives the results in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-5


def listed():
    return [
        # a training step on one small batch of short clips: launches, hardly any work
        dict(name="norm_clips", kind="norm", B=40, T=32, H=1, D=512, dtype="f16", lengths="clips", center=True, bias=True,
             residual=False, fused=False, train=True),
        # documents that nearly fill their blocks, the norm in front of a layer with the residual stream's sum
        dict(name="norm_documents", kind="norm", B=8, T=4096, H=1, D=4096, dtype="bf16", lengths="full", center=True, bias=True,
             residual=True, fused=False, train=True),
        # queries and keys of one layer, every head by itself, where they lie in the projection's result
        dict(name="norm_heads", kind="norm", B=8, T=3000, H=20, D=128, dtype="bf16", lengths="pareto", center=False, bias=False,
             residual=False, fused=True, train=True),
        # rows of an odd number of floats, no gradient
        dict(name="norm_odd", kind="norm", B=24, T=777, H=1, D=1537, dtype="f32", lengths="uniform", center=True, bias=True,
             residual=True, fused=False, train=False),
        # half of a projection's result, recordings of heavy-tailed length
        dict(name="conv_recordings", kind="conv", B=16, T=3000, D=4096, K=4, dtype="bf16", lengths="pareto", silu=True, bias=True,
             state=False, fused=True, train=True),
        # an odd number of float features in blocks of 777, streams that go on
        dict(name="conv_odd", kind="conv", B=24, T=777, D=333, K=3, dtype="f32", lengths="uniform", silu=False, bias=False,
             state=True, fused=False, train=True),
        # one new frame of 256 streams
        dict(name="conv_step", kind="conv", B=256, T=1, D=4096, K=4, dtype="bf16", lengths="clips", silu=True, bias=True,
             state=True, fused=True, train=False),
        # a training step on short clips: latency
        dict(name="scan_clips", kind="scan", B=40, T=32, D=256, N=16, G=1, dtype="f16", lengths="clips", z=True, softplus=True,
             state=False, fused=True, train=True),
        # two prompts of a serving program, which goes on from their states
        dict(name="scan_prompt", kind="scan", B=2, T=4096, D=2048, N=16, G=1, dtype="bf16", lengths="full", z=True, softplus=True,
             state=True, fused=True, train=False),
        # training on documents: the vector units' work
        dict(name="scan_documents", kind="scan", B=8, T=4096, D=4096, N=16, G=1, dtype="bf16", lengths="full", z=True,
             softplus=True, state=False, fused=True, train=True),
        # two groups of 100 float channels, 24 states, steps given as they are, streams that go on
        dict(name="scan_odd", kind="scan", B=6, T=777, D=200, N=24, G=2, dtype="f32", lengths="uniform", z=False, softplus=False,
             state=True, fused=False, train=True),
        # one new frame of 256 streams: the states are read and written, nothing else
        dict(name="scan_step", kind="scan", B=256, T=1, D=4096, N=16, G=1, dtype="bf16", lengths="clips", z=True, softplus=True,
             state=True, fused=True, train=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MIXES = ["clips", "uniform", "pareto", "video", "speech", "zipf", "full"]


def draw(rng):
    kind = rng.choice(["norm", "norm", "conv", "conv", "scan", "scan", "scan"])
    lengths = rng.choice(MIXES)
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    yes = lambda p: rng.random() < p
    if kind == "norm":
        if yes(0.4):
            H, D = rng.choice([2, 5, 6, 10, 16, 40]), rng.choice([64, 128, rng.randint(1, 256)])
        else:
            H, D = 1, rng.choice([_log(rng, 1, 512), 16 * _log(rng, 1, 512), _log(rng, 64, 16384)])
        T = _log(rng, 1, 4096)
        elements = math.exp(rng.uniform(math.log(1e4), math.log(6e7)))
        center = yes(0.6)
        return dict(kind=kind, B=int(min(4096, max(1, round(elements / (T * H * D))))), T=T, H=H, D=D, dtype=dtype,
                    lengths=lengths, center=center, bias=center and yes(0.7), residual=yes(0.5), fused=yes(0.4), train=yes(0.6))
    D = rng.choice([_log(rng, 1, 64), 16 * _log(rng, 1, 256), _log(rng, 64, 4096)])
    step = yes(0.3)
    if kind == "conv":
        T = 1 if step else _log(rng, 2, 6000)
        elements = math.exp(rng.uniform(math.log(1e4), math.log(1e8)))
        return dict(kind=kind, B=int(min(4096, max(1, round(elements / (T * D))))), T=T, D=D, K=rng.choice([2, 3, 4, 4, 4, 5, 8]),
                    dtype=dtype, lengths=lengths, silu=yes(0.7), bias=yes(0.7), state=step or yes(0.4), fused=yes(0.5),
                    train=not step and yes(0.7))
    N = rng.choice([16, 16, 8, rng.randint(1, 32), 64])
    G = rng.choice([g for g in (1, 1, 2, 4, 8) if D % g == 0])
    T = 1 if step else _log(rng, 2, 6000)
    elements = math.exp(rng.uniform(math.log(1e5), math.log((1.6e7 if step else 6e8) / N)))
    return dict(kind=kind, B=int(min(4096, max(1, round(elements / (T * D))))), T=T, D=D, N=N, G=G, dtype=dtype, lengths=lengths,
                z=yes(0.7), softplus=yes(0.7), state=step or yes(0.4), fused=yes(0.5), train=not step and yes(0.6))


# ---------------------------------------------------------------- inputs


def draw_lengths(mix, n, t_blk, g):
    """int64[n] in [1, t_blk], the mixes that the packer itself is measured on."""
    if mix == "clips":                   # short clips of a few to t_blk frames
        x = g.integers(max(1, t_blk // 16), t_blk, size=n, endpoint=True)
    elif mix == "uniform":
        x = g.integers(1, t_blk, size=n, endpoint=True)
    elif mix == "pareto":                # many short, few very long
        x = np.floor(8.0 * (1.0 + g.pareto(1.5, size=n)))
    elif mix == "video":                 # median a tenth of the block
        x = np.rint(g.lognormal(math.log(max(1.0, t_blk / 10.0)), 1.0, size=n))
    elif mix == "speech":                # uniform from a thirtieth of the block
        x = g.integers(max(1, t_blk // 30), t_blk, size=n, endpoint=True)
    elif mix == "zipf":                  # documents: half of them a token or two, a sixth fill a block
        x = g.zipf(1.2, size=n)
    elif mix == "full":                  # nearly every sequence fills its block
        x = t_blk - np.minimum(g.geometric(0.3, size=n) - 1, t_blk - 1)
    else:
        raise KeyError(mix)
    return np.clip(x, 1, t_blk).astype(np.int64)


def _fill(case):
    """Sequences of the case's mix laid one after another into its B blocks: block, first slot and length of each.  Where
    states are handed on, the last one of a block goes on to its end, and in the next block."""
    B, T = case["B"], case["T"]
    g = np.random.Generator(np.random.PCG64([17, B, T]))
    block, first, length, b, at = [], [], [], 0, 0
    while True:
        for n in draw_lengths(case["lengths"], 256, T, g).tolist():
            if at + n > T:
                b, at = b + 1, 0
            if b == B:
                block, first, length = np.asarray(block), np.asarray(first), np.asarray(length)
                if case.get("state"):
                    last = np.append(block[1:] != block[:-1], True)
                    length[last] = T - first[last]
                return block, first, length
            block.append(b)
            first.append(at)
            length.append(n)
            at += n


class State:
    """What a program holds between calls."""


def _tables(s, case, seed):
    """The start table as the packer leaves it, with the blocks in an order of the seed's."""
    block, first, length = _fill(case)
    B, T = case["B"], case["T"]
    block = np.random.Generator(np.random.PCG64([18, seed])).permutation(B)[block]
    slot0 = torch.from_numpy(block * T + first).cuda()
    count = torch.from_numpy(length).cuda()
    start = torch.cumsum(count, 0) - count
    frame = torch.arange(int(length.sum()), device="cuda") - torch.repeat_interleave(start, count)
    slot = frame + torch.repeat_interleave(slot0, count)
    s.frame_idx = torch.full((B * T,), -1, dtype=torch.int32, device="cuda")
    s.frame_idx[slot] = frame.to(torch.int32)
    s.frame_idx = s.frame_idx.view(B, T)
    s.valid = (s.frame_idx >= 0).to(torch.uint8)
    s.reset = (s.frame_idx == 0).to(torch.uint8)
    if case.get("state"):                                        # streams that go on: no start at the first slot
        s.reset[:, 0] = 0


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=DTYPES[dtype], device="cuda").normal_(generator=g)


def _real(shape, g, mean=0.0, std=1.0):
    return torch.empty(shape, device="cuda").normal_(mean, std, generator=g)


def prepare(case, seed):
    s = State()
    s.case, kind, dtype = case, case["kind"], case["dtype"]
    B, T, D = case["B"], case["T"], case["D"]
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 31)
    _tables(s, case, seed)
    if kind == "norm":
        H = case["H"]
        # a stream with some mean, in its own memory or the first heads of a projection's result
        s.x = _normal((B, T, H + 2, D), dtype, g)[:, :, :H] if case["fused"] else _normal((B, T, H, D), dtype, g)
        s.x.mul_(1.5).add_(0.25)
        s.weight = _real((D,), g, 1.0, 0.2)
        s.bias = _real((D,), g, 0.0, 0.2) if case["bias"] else None
        s.residual = _normal((B, T, H, D), dtype, g) if case["residual"] else None
        if case["train"]:
            s.dout = _normal((B, T, H, D), dtype, g)
            s.dsum = _normal((B, T, H, D), dtype, g) if case["residual"] else None
        return s
    if kind == "conv":
        K = case["K"]
        s.x = _normal((B, T, 2, D), dtype, g)[:, :, 0] if case["fused"] else _normal((B, T, D), dtype, g)
        s.weight = _real((D, K), g, 0.0, K ** -0.5)
        s.bias = _real((D,), g, 0.0, 0.2) if case["bias"] else None
        s.state = _normal((B, K - 1, D), dtype, g) if case["state"] else None
        if case["train"]:
            s.dout = _normal((B, T, D), dtype, g)
            s.dstate = _normal((B, K - 1, D), dtype, g) if case["state"] else None
        return s
    N, G = case["N"], case["G"]
    s.z = None
    if case["fused"]:                                            # steps, B and C of one projection; x and z of another one
        xz = _normal((B, T, 2, D), dtype, g)
        s.x = xz[:, :, 0]
        s.z = xz[:, :, 1] if case["z"] else None
        bc = _normal((B, T, 2, G, N), dtype, g)
        s.b, s.c = bc[:, :, 0], bc[:, :, 1]
    else:
        s.x = _normal((B, T, D), dtype, g)
        s.z = _normal((B, T, D), dtype, g) if case["z"] else None
        s.b, s.c = (_normal((B, T, G, N), dtype, g) for _ in range(2))
    # rates of 1 .. N and a little noise, steps from a thousandth to a tenth
    s.a = -(1.0 + torch.arange(N, device="cuda")) * torch.exp(_real((D, N), g, 0.0, 0.1))
    steps = torch.exp(torch.empty((D,), device="cuda").uniform_(math.log(1e-3), math.log(0.1), generator=g))
    if case["softplus"]:
        s.dt_bias = steps + torch.log(-torch.expm1(-steps))
        s.dt = _normal((B, T, D), dtype, g).mul_(0.5)
    else:
        s.dt_bias = None
        s.dt = (steps * torch.exp(_real((B, T, D), g, 0.0, 0.5))).to(DTYPES[dtype])
    s.skip = _real((D,), g, 1.0, 0.1)
    s.h0 = _real((B, D, N), g) if case["state"] else None
    if case["train"]:
        s.dout = _normal((B, T, D), dtype, g)
        s.dstate = _real((B, D, N), g) if case["state"] else None
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2310_10879_amd import bload
    c, kind = s.case, s.case["kind"]
    if kind == "norm":
        got = bload.bload_layer_norm(s.x, s.weight, s.bias, residual=s.residual, valid=s.valid, eps=EPS, center=c["center"],
                                     training=c["train"])
        got = list(got) if isinstance(got, tuple) else [got]
        if not c["train"]:
            return got
        stats = got.pop()
        dx, dweight, dbias = bload.bload_layer_norm_backward(s.dout, got[1] if c["residual"] else s.x, stats, s.weight,
                                                             valid=s.valid, dsum=s.dsum, center=c["center"])
        return got + [dx, dweight] + ([dbias] if c["bias"] else [])
    if kind == "conv":
        y, state = bload.bload_segment_conv(s.x, s.weight, s.reset, s.valid, bias=s.bias, silu=c["silu"], state_in=s.state)
        if not c["train"]:
            return [y, state]
        dx, dweight, dbias, dstate = bload.bload_segment_conv_backward(s.dout, s.x, s.weight, s.reset, s.valid, bias=s.bias,
                                                                       silu=c["silu"], state_in=s.state, dstate=s.dstate)
        return [y, state, dx, dweight] + ([dbias] if c["bias"] else []) + ([dstate] if c["state"] else [])
    args = dict(skip=s.skip, z=s.z, dt_bias=s.dt_bias, softplus=c["softplus"], h0=s.h0)
    if not c["train"]:
        return list(bload.bload_selective_scan(s.x, s.dt, s.a, s.b, s.c, s.reset, s.valid, **args))
    y, state, saved = bload.bload_selective_scan(s.x, s.dt, s.a, s.b, s.c, s.reset, s.valid, **args, training=True)
    grads = bload.bload_selective_scan_backward(s.dout, s.x, s.dt, s.a, s.b, s.c, s.reset, s.valid, saved, **args, dstate=s.dstate)
    return [y, state] + [t for t in grads if t is not None]


def _run_plain(s):
    return {"norm": _plain_norm, "conv": _plain_conv, "scan": _plain_scan}[s.case["kind"]](s)


def _plain_norm(s):
    c, t = s.case, s.x.dtype
    live = s.valid.bool()[:, :, None, None]
    x = s.x.float()
    if c["residual"]:
        x = (x + s.residual.float()).masked_fill_(~live, 0.0)
        total = x.to(t)
        x = total.float()                                        # the stream that is handed on is what is normalised
    mean = x.mean(3, keepdim=True) if c["center"] else 0.0
    x = x - mean
    r = torch.rsqrt((x * x).mean(3, keepdim=True) + EPS)
    x = x * r
    y = x * s.weight
    if c["bias"]:
        y = y + s.bias
    out = [y.masked_fill_(~live, 0.0).to(t)] + ([total] if c["residual"] else [])
    if not c["train"]:
        return out
    dy = s.dout.float().masked_fill_(~live, 0.0)
    g = dy * s.weight
    dx = g - x * (g * x).mean(3, keepdim=True)
    if c["center"]:
        dx = dx - g.mean(3, keepdim=True)
    dx = dx * r
    if c["residual"]:
        dx = dx + s.dsum.float()
    out += [dx.masked_fill_(~live, 0.0).to(t), (dy * x).masked_fill_(~live, 0.0).sum((0, 1, 2))]
    return out + ([dy.sum((0, 1, 2))] if c["bias"] else [])


def _goes_on(s):
    """True where a slot goes on from the one in front of it (the first one: from the state handed in)."""
    before = torch.cat([torch.full_like(s.valid[:, :1], bool(s.case["state"])), s.valid[:, :-1]], 1)
    return (s.valid == 1) & (s.reset == 0) & (before == 1)


def _taps(s):
    """bool[B, T] for each tap j: does slot t see the input of j slots before it; and what the state keeps behind the last."""
    K, T = s.case["K"], s.case["T"]
    age = s.frame_idx.long()                                     # slots of its sequence in front of it
    if s.case["state"]:                                          # (the first sequence of a block has K - 1 more)
        first = torch.cumsum(1 - _goes_on(s).long(), 1) == 0
        age = torch.where(first, torch.arange(T, device="cuda") + K - 1, age)
    live = s.valid == 1
    last = [(live & (age >= K - 2 - i))[:, -1] for i in range(K - 1)]
    return [live & (age >= j) for j in range(K)], last


def _plain_conv(s):
    c, t = s.case, s.x.dtype
    B, T, D, K = c["B"], c["T"], c["D"], c["K"]
    x = s.x.float()
    front = torch.zeros((B, K - 1, D), device="cuda") if s.state is None else s.state.float()
    x = torch.cat([front, x], 1)
    taps, last = _taps(s)
    seen = lambda j: x[:, K - 1 - j:K - 1 - j + T] * taps[j][:, :, None]
    p = torch.zeros((B, T, D), device="cuda")
    for j in range(K):
        p += s.weight[:, K - 1 - j] * seen(j)
    if c["bias"]:
        p += s.bias * taps[0][:, :, None]
    sig = torch.sigmoid(p)
    y = p * sig if c["silu"] else p
    state = [x[:, T + i] * keep[:, None] for i, keep in enumerate(last)]
    out = [y.to(t), torch.stack(state, 1).to(t)]
    if not c["train"]:
        return out
    dp = s.dout.float() * taps[0][:, :, None]
    if c["silu"]:
        dp = dp * sig * (1.0 + p * (1.0 - sig))
    dx = torch.zeros_like(x)
    dw = torch.empty_like(s.weight)
    for j in range(K):
        dx[:, K - 1 - j:K - 1 - j + T] += s.weight[:, K - 1 - j] * dp * taps[j][:, :, None]
        dw[:, K - 1 - j] = (dp * seen(j)).sum((0, 1))
    if s.dstate is not None:
        for i, keep in enumerate(last):
            dx[:, T + i] += s.dstate[:, i].float() * keep[:, None]
    out += [dx[:, K - 1:].to(t), dw] + ([dp.sum((0, 1))] if c["bias"] else [])
    return out + ([dx[:, :K - 1].to(t)] if c["state"] else [])


def _recurrence(a, x):
    """h[:, t] = a[:, t] * h[:, t - 1] + x[:, t] by doubling: after step d, h holds the part of the last 2 d frames."""
    d = 1
    while d < x.shape[1]:
        x = torch.cat([x[:, :d], x[:, d:] + a[:, d:] * x[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return x


def _plain_scan(s):
    """A slab of channels at a time, so that [B, T, slab, N] stays around two gigabytes."""
    c, t = s.case, s.x.dtype
    B, T, D, N, G = c["B"], c["T"], c["D"], c["N"], c["G"]
    on, live = _goes_on(s)[:, :, None].float(), (s.valid == 1)[:, :, None].float()
    per = D // G
    slab = max(1, min(per, int(5e8 / (B * T * N))))
    parts = []
    db, dc = (torch.zeros((B, T, G, N), device="cuda") for _ in range(2))
    for group in range(G):
        b, cc = (v[:, :, group].float()[:, :, None] for v in (s.b, s.c))
        for lo in range(group * per, (group + 1) * per, slab):
            at = slice(lo, min(lo + slab, (group + 1) * per))
            x, v = s.x[:, :, at].float() * live, s.dt[:, :, at].float()
            if s.dt_bias is not None:
                v = v + s.dt_bias[at]
            delta = torch.log1p(torch.exp(-v.abs())) + v.clamp(min=0.0) if c["softplus"] else v
            delta = delta * live
            rate = s.a[at]
            decay = torch.exp(delta[..., None] * rate) * on[..., None]
            u = (delta * x)[..., None] * b
            if s.h0 is not None:
                u[:, 0] += decay[:, 0] * s.h0[:, at]
            h = _recurrence(decay, u)
            del u
            y = (h * cc).sum(3) + s.skip[at] * x
            if c["z"]:
                z = s.z[:, :, at].float() * live
                sig = torch.sigmoid(z)
                out = y * z * sig
            else:
                out = y
            part = [out.to(t), h[:, -1].clone()]
            if c["train"]:
                dy = s.dout[:, :, at].float() * live
                dz = None
                if c["z"]:
                    dz = (dy * y * sig * (1.0 + z * (1.0 - sig))).to(t)
                    dy = dy * z * sig
                dc[:, :, group] += (dy[..., None] * h).sum(2)
                dh = dy[..., None] * cc
                if s.dstate is not None:
                    dh[:, -1] += s.dstate[:, at] * live[:, -1:]
                nxt = torch.cat([decay[:, 1:], torch.zeros_like(decay[:, :1])], 1)
                g = _recurrence(nxt.flip(1), dh.flip(1)).flip(1)
                del nxt, dh
                db[:, :, group] += (g * (delta * x)[..., None]).sum(2)
                q = (g * b).sum(3)
                before = torch.cat([torch.zeros_like(h[:, :1]) if s.h0 is None else s.h0[:, None, at], h[:, :-1]], 1)
                g *= decay
                dh0 = g[:, 0].clone()
                g *= before
                del before
                ddt = (g * rate).sum(3) + x * q
                da = (g * delta[..., None]).sum((0, 1))
                if c["softplus"]:
                    ddt = ddt * torch.sigmoid(v)
                ddt = ddt * live
                part += [(delta * q + s.skip[at] * dy).to(t), ddt.to(t), da, (dy * x).sum((0, 1)), dz, ddt.sum((0, 1)), dh0]
            parts.append(part)
    joined = [torch.cat([p[i] for p in parts], dim) if parts[0][i] is not None else None
              for i, dim in zip(range(len(parts[0])), (2, 1, 2, 2, 0, 0, 2, 0, 1))]
    return joined[:2] if not c["train"] else _scan_outputs(s, *joined[:5], db.to(t), dc.to(t), *joined[5:])


def _scan_outputs(s, out, state, dx, ddt, da, db, dc, dskip, dz, dbias, dh0):
    """Results and gradients by x, dt, A, B, C, the skip, z, the bias of dt and the state, of what the case has."""
    return [out, state, dx, ddt, da, db, dc, dskip] + ([dz] if s.z is not None else []) + \
        ([dbias] if s.dt_bias is not None else []) + ([dh0] if s.h0 is not None else [])


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    B, T, D, kind, e = case["B"], case["T"], case["D"], case["kind"], BYTES[case["dtype"]]
    frames, slots, train = float(_fill(case)[2].sum()), B * T, case["train"]
    if kind == "norm":
        H, both = case["H"], 2 if case["residual"] else 1
        row = e * H * D
        moved = row * both * (frames + slots) + slots + 4 * D * (2 if case["bias"] else 1)
        if train:                                                # (x, or the sum, is in hand from the forward pass)
            moved += row * (both * frames + slots) + 4 * D * (2 if case["bias"] else 1)
        return {"bytes": moved, "flops": (20 if train else 8) * frames * H * D}
    if kind == "conv":
        K = case["K"]
        state = e * B * (K - 1) * D
        moved = e * D * (frames + slots) + 2 * slots + 4 * D * (K + 1) + state * (2 if case["state"] else 1)
        if train:
            moved += e * D * (frames + slots) + 4 * D * (K + 1) + state * (2 if case["state"] else 0)
        return {"bytes": moved, "flops": (6 * K + 12 if train else 2 * K + 4) * frames * D}
    N, G = case["N"], case["G"]
    ins, state = 3 if case["z"] else 2, 4 * B * D * N
    moved = e * D * (ins * frames + slots) + 2 * e * G * N * frames + 2 * slots + 4 * D * (N + 2) + state * (2 if case["state"] else 1)
    if train:
        moved += e * D * (frames + ins * slots) + 2 * e * G * N * slots + 4 * D * (N + 2) + state * (2 if case["state"] else 0)
    return {"bytes": moved, "flops": (21 if train else 7) * frames * D * N}


# ---------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "conv": _exact_conv, "scan": _exact_scan}[case["kind"]](s)


def _exact_norm(s):
    """The gradients from torch's own differentiation."""
    c = s.case
    live = s.valid.bool()
    x = s.x.double()[live]                                       # [rows, H, D]
    total = None
    if c["residual"]:
        total = (s.x.double() + s.residual.double())[live]
        # what goes on is the rounded sum, and that is normalised
        x = (s.x.float() + s.residual.float())[live].to(s.x.dtype).double()
    x.requires_grad_(c["train"])
    weight = s.weight.double().requires_grad_(c["train"])
    bias = s.bias.double().requires_grad_(c["train"]) if c["bias"] else None
    if c["center"]:
        y = (x - x.mean(2, keepdim=True)) / torch.sqrt(x.var(2, unbiased=False, keepdim=True) + EPS)
    else:
        y = x / torch.sqrt(x.square().mean(2, keepdim=True) + EPS)
    y = y * weight
    if bias is not None:
        y = y + bias

    def spread(rows):
        full = torch.zeros(s.x.shape, dtype=torch.float64, device="cuda")
        full[live] = rows
        return full
    out = [spread(y.detach())] + ([spread(total)] if c["residual"] else [])
    if not c["train"]:
        return out
    y.backward(s.dout.double()[live])
    dx = x.grad + s.dsum.double()[live] if c["residual"] else x.grad
    return out + [spread(dx), weight.grad] + ([bias.grad] if c["bias"] else [])


def _exact_conv(s):
    """Every tap's slot by its index; the gradients from torch's own differentiation."""
    c = s.case
    B, T, D, K = c["B"], c["T"], c["D"], c["K"]
    on = _goes_on(s)
    leaf = lambda v: None if v is None else v.double().requires_grad_(c["train"])
    x, weight, bias, state = leaf(s.x), leaf(s.weight), leaf(s.bias), leaf(s.state)
    front = torch.zeros((B, K - 1, D), dtype=torch.float64, device="cuda") if state is None else state
    rows = torch.cat([front, x], 1)
    reach = (s.valid == 1)[:, :, None].double()                  # does slot t look back over j slots
    live = reach
    p = 0.0 if bias is None else bias * live
    goes = torch.cat([torch.ones((B, K - 1), dtype=torch.float64, device="cuda"), on.double()], 1)[:, :, None]
    for j in range(K):
        p = p + rows[:, K - 1 - j:K - 1 - j + T] * (reach * weight[:, K - 1 - j])
        reach = reach * goes[:, K - 1 - j:K - 1 - j + T]
    y = p * torch.sigmoid(p) if c["silu"] else p
    left, keep = [], live[:, -1]
    for i in range(K - 1):                                       # the last K - 1 inputs, as far as the last sequence has them
        left.append(rows[:, K - 2 + T - i] * keep)
        keep = keep * goes[:, K - 2 + T - i]
    left = torch.stack(left[::-1], 1)
    out = [y.detach(), left.detach()]
    if not c["train"]:
        return out
    torch.autograd.backward([y] + ([left] if c["state"] else []), [s.dout.double()] + ([s.dstate.double()] if c["state"] else []))
    return out + [v.grad for v in (x, weight, bias, state) if v is not None]


def _exact_scan(s):
    """Frame by frame, the channels of a group side by side."""
    c = s.case
    B, T, D, N, G = c["B"], c["T"], c["D"], c["N"], c["G"]
    if T * B * D * N > 2.2e9:
        return None
    on = _goes_on(s).double()[:, :, None, None]
    live = (s.valid == 1).double()[:, :, None]
    wide = lambda v: v.double().repeat_interleave(D // G, dim=1)          # [B, G, N] -> [B, D, N]
    x = s.x.double() * live
    v = s.dt.double() + (0.0 if s.dt_bias is None else s.dt_bias.double())
    delta = (torch.logaddexp(v, torch.zeros_like(v)) if c["softplus"] else v) * live
    a = s.a.double()
    skip = s.skip.double()
    hs = torch.empty((T + 1, B, D, N), dtype=torch.float64, device="cuda")
    hs[0] = 0.0 if s.h0 is None else s.h0.double()
    y = torch.empty((B, T, D), dtype=torch.float64, device="cuda")
    for t in range(T):
        hs[t + 1] = torch.exp(delta[:, t, :, None] * a) * on[:, t] * hs[t] + (delta[:, t] * x[:, t])[..., None] * wide(s.b[:, t])
        y[:, t] = (hs[t + 1] * wide(s.c[:, t])).sum(2)
    y += skip * x
    z = s.z.double() * live if c["z"] else None
    gate = 1.0 if z is None else z * torch.sigmoid(z)
    out, state = y * gate, hs[T].clone()
    if not c["train"]:
        return [out, state]
    dout = s.dout.double() * live
    dy = dout * gate
    dz = None if z is None else dout * y * torch.sigmoid(z) * (1.0 + z * (1.0 - torch.sigmoid(z)))
    g = torch.zeros((B, D, N), dtype=torch.float64, device="cuda") if s.dstate is None else s.dstate.double() * live[:, -1, :, None]
    q, ddt = torch.empty_like(y), torch.empty_like(y)
    da = torch.zeros_like(a)
    db, dc = (torch.empty((B, T, G, N), dtype=torch.float64, device="cuda") for _ in range(2))
    for t in range(T - 1, -1, -1):
        g = g + dy[:, t, :, None] * wide(s.c[:, t])
        dc[:, t] = (dy[:, t, :, None] * hs[t + 1]).view(B, G, D // G, N).sum(2)
        db[:, t] = ((delta[:, t] * x[:, t])[..., None] * g).view(B, G, D // G, N).sum(2)
        q[:, t] = (g * wide(s.b[:, t])).sum(2)
        g = g * torch.exp(delta[:, t, :, None] * a) * on[:, t]
        p = g * hs[t]
        ddt[:, t] = (p * a).sum(2)
        da += (p * delta[:, t, :, None]).sum(0)
    dx = delta * q + skip * dy
    ddt = (ddt + x * q) * live
    if c["softplus"]:
        ddt = ddt * torch.sigmoid(v)
    return _scan_outputs(s, out, state, dx, ddt, da, db, dc, (dy * x).sum((0, 1)), dz, ddt.sum((0, 1)), g)
