"""Performance cases of the operators that train and serve a sequence model on packed blocks.

The packer leaves blocks ``[B, T, ...]`` of whole sequences with a start table.  A case is a dict of
plain values; ``kind`` says which operator one pass goes through:

    attention  attention inside the sequences of the blocks: the mask from the start table, the forward
               pass and, where ``train`` is set, the backward pass
    decode     one query per sequence over the packed blocks as a cache of keys and values
    gated      the recurrence h = gate * h_prev + x with the blocks' resets, forward and backward
    step       the same recurrence for one new frame of every stream, state in and state out
    rotary     rotary positions from the frame numbers, forward or (``inverse``) the gradient's rotation

``lengths`` names the mix of sequence lengths (see ``draw_lengths``).  The lengths belong to the case
and the seed draws the order of the blocks and the payload, so that every seed fills tensors of the
same shape.  With ``own`` false a pass is plain torch in 32 bits (64 for angles), with ``own`` true it
makes the calls of ``paper_2310_10879_amd.bload``.  ``exact`` gives the results in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # a training step on one small batch of short clips: all launches, hardly any work
        dict(name="attention_clips", kind="attention", B=40, T=32, Hq=4, Hkv=4, D=64, dtype="f16", lengths="clips",
             causal=True, prefix=False, cap=0.0, slopes=False, fused=True, train=True),
        # recordings of heavy-tailed length: dozens of short sequences and a few long ones in each block
        dict(name="attention_recordings", kind="attention", B=16, T=3000, Hq=16, Hkv=16, D=128, dtype="f16",
             lengths="pareto", causal=True, prefix=False, cap=0.0, slopes=False, fused=True, train=True),
        # documents that nearly fill their blocks, grouped heads: the matrix products are all that counts
        dict(name="attention_documents", kind="attention", B=8, T=4096, Hq=32, Hkv=8, D=128, dtype="bf16",
             lengths="full", causal=True, prefix=False, cap=0.0, slopes=False, fused=False, train=True),
        # heads of 37 elements in blocks of 777: nothing is a multiple of anything; capped scores, a bias
        # by distance and a prefix that all of a sequence sees
        dict(name="attention_odd", kind="attention", B=24, T=777, Hq=6, Hkv=2, D=37, dtype="bf16", lengths="uniform",
             causal=True, prefix=True, cap=30.0, slopes=True, fused=True, train=True),
        # log-mel frames of 80 floats, every frame sees its whole recording, no gradient
        dict(name="attention_mel", kind="attention", B=12, T=3000, Hq=4, Hkv=4, D=80, dtype="f32", lengths="speech",
             causal=False, prefix=False, cap=0.0, slopes=False, fused=False, train=False),
        # a handful of streams ask for their next frame: latency
        dict(name="decode_few", kind="decode", B=4, T=600, Hq=16, Hkv=4, D=64, dtype="f16", lengths="video", cap=0.0,
             slopes=False, fused=False),
        # long streams, grouped heads: the cache is read once, nothing else
        dict(name="decode_long", kind="decode", B=32, T=32768, Hq=32, Hkv=8, D=128, dtype="bf16", lengths="speech",
             cap=50.0, slopes=False, fused=True),
        # 2048 half-precision features with many starts in each block
        dict(name="gated_features", kind="gated", B=48, T=3000, D=2048, dtype="f16", lengths="pareto", state=False),
        # one block of log-mel frames with carried state: few lanes, a long way
        dict(name="gated_mel", kind="gated", B=8, T=3000, D=80, dtype="f32", lengths="speech", state=True),
        # the recurrence of 256 streams, one new frame each
        dict(name="gated_step", kind="step", B=256, T=1, D=2048, dtype="bf16"),
        # queries and keys of one layer, rotated together where they lie in the projection's result
        dict(name="rotary_heads", kind="rotary", B=16, T=4096, H=40, D=128, rot=128, layout="half", dtype="bf16",
             lengths="zipf", far=0, scaled=False, fused=True, inverse=False),
        # a quarter of an odd head, neighbours paired, positions of a long stream with scaled frequencies: the gradient
        dict(name="rotary_far", kind="rotary", B=24, T=777, H=6, D=74, rot=18, layout="interleaved", dtype="f32",
             lengths="uniform", far=1 << 20, scaled=True, fused=False, inverse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MIXES = ["clips", "uniform", "pareto", "video", "speech", "zipf", "full"]


def draw(rng):
    kind = rng.choice(["attention"] * 4 + ["decode"] * 2 + ["gated"] * 3 + ["step", "rotary", "rotary"])
    lengths = rng.choice(MIXES)
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    Hkv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
    D = rng.choice([64, 128, 8 * rng.randint(1, 16), rng.randint(1, 128)])
    if kind == "attention":
        T = _log(rng, 16, 4096)
        most = 2.0e9 / 4 if dtype == "f32" else 2.0e9          # B Hq T^2; the largest listed has 4.3e9
        B = int(math.exp(rng.uniform(0.0, math.log(max(1.0, min(64.0, most / (Hkv * group * T * T)))))))
        causal = rng.random() < 0.7
        return dict(kind=kind, B=B, T=T, Hq=Hkv * group, Hkv=Hkv, D=D, dtype=dtype, lengths=lengths, causal=causal,
                    prefix=causal and rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                    slopes=rng.random() < 0.3, fused=rng.random() < 0.5, train=rng.random() < 0.7)
    if kind == "decode":
        T = _log(rng, 16, 32768)
        slots = int(math.exp(rng.uniform(math.log(64.0), math.log(2.5e8 / (Hkv * D * BYTES[dtype])))))
        if lengths in ("zipf", "pareto", "clips"):              # (the plain form pads every sequence to the longest)
            lengths = "speech"
        return dict(kind=kind, B=max(1, min(512, slots // T)), T=T, Hq=Hkv * group, Hkv=Hkv, D=D, dtype=dtype,
                    lengths=lengths, cap=rng.choice([0.0, 0.0, 50.0]), slopes=rng.random() < 0.3,
                    fused=rng.random() < 0.5)
    D = rng.choice([_log(rng, 1, 64), 16 * _log(rng, 1, 128), _log(rng, 64, 4096)])
    if kind == "gated":
        T = _log(rng, 2, 6000)
        elements = math.exp(rng.uniform(math.log(1e4), math.log(1.2e8)))
        return dict(kind=kind, B=int(min(4096, max(1, round(elements / (T * D))))), T=T, D=D, dtype=dtype,
                    lengths=lengths, state=rng.random() < 0.5)
    if kind == "step":
        return dict(kind=kind, B=_log(rng, 1, 4096), T=1, D=D, dtype=dtype)
    H, D = rng.choice([1, 2, 6, 10, 16, 40]), rng.choice([64, 128, 2 * rng.randint(1, 64)])
    T = _log(rng, 16, 4096)
    elements = math.exp(rng.uniform(math.log(1e4), math.log(3e8)))
    return dict(kind=kind, B=int(min(1024, max(1, round(elements / (T * H * D))))), T=T, H=H, D=D,
                rot=D if rng.random() < 0.5 else 2 * rng.randint(1, D // 2), layout=rng.choice(["half", "interleaved"]),
                dtype=dtype, lengths=lengths, far=rng.choice([0, 0, 1 << 16, 1 << 24]), scaled=rng.random() < 0.5,
                fused=rng.random() < 0.5, inverse=rng.random() < 0.5)


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
    """Sequences of the case's mix laid one after another into its B blocks: block, first slot and length of each."""
    B, T = case["B"], case["T"]
    g = np.random.Generator(np.random.PCG64([17, B, T]))
    block, first, length, b, at = [], [], [], 0, 0
    while True:
        for n in draw_lengths(case["lengths"], 256, T, g).tolist():
            if at + n > T:
                b, at = b + 1, 0
            if b == B:
                return np.asarray(block), np.asarray(first), np.asarray(length)
            block.append(b)
            first.append(at)
            length.append(n)
            at += n


class State:
    """What a program holds between calls."""


def _tables(s, case, seed):
    """The start table as the packer leaves it, with the blocks in an order of the seed's."""
    block, first, length = _fill(case)
    B, T, n = case["B"], case["T"], len(length)
    block = np.random.Generator(np.random.PCG64([18, seed])).permutation(B)[block]
    s.n_seq = n
    s.block_of_seq, s.offset_of_seq, s.lengths = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (block, first, length))
    slot0 = torch.from_numpy(block * T + first).cuda()
    count = torch.from_numpy(length).cuda()
    start = torch.cumsum(count, 0) - count
    frame = torch.arange(int(length.sum()), device="cuda") - torch.repeat_interleave(start, count)
    slot = frame + torch.repeat_interleave(slot0, count)
    s.seq_id = torch.full((B * T,), -1, dtype=torch.int32, device="cuda")
    s.seq_id[slot] = torch.repeat_interleave(torch.arange(n, dtype=torch.int32, device="cuda"), count)
    s.frame_idx = torch.full((B * T,), -1, dtype=torch.int32, device="cuda")
    s.frame_idx[slot] = frame.to(torch.int32)
    s.reset = torch.zeros(B * T, dtype=torch.uint8, device="cuda")
    s.reset[slot0] = 1
    s.valid = (s.seq_id >= 0).to(torch.uint8)
    for name in ("seq_id", "frame_idx", "reset", "valid"):
        setattr(s, name, getattr(s, name).view(B, T))


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=DTYPES[dtype], device="cuda").normal_(generator=g)


def _slopes(case, device="cuda"):
    """A bias by distance: 2^-1 ... 2^-8 over the heads."""
    H = case["Hq"]
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=device)


def _frequencies(case):
    """Radians per frame of each pair of elements; where scaled, the slow ones divided by 8 and a ramp between."""
    rot = case["rot"]
    f = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if case["scaled"]:
        turns = 4096.0 * f / (2.0 * math.pi)                     # turns over the length trained on
        keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * (keep + (1.0 - keep) / 8.0)
    return torch.from_numpy(f.astype(np.float32)).cuda()


def prepare(case, seed):
    s = State()
    s.case, kind, dtype = case, case["kind"], case["dtype"]
    B, T, D = case["B"], case["T"], case["D"]
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 29)
    if kind != "step":
        _tables(s, case, seed)
    if kind == "attention":
        Hq, Hkv = case["Hq"], case["Hkv"]
        if case["fused"]:                                        # one projection's result, cut by heads
            qkv = _normal((B, T, Hq + 2 * Hkv, D), dtype, g)
            s.q, s.k, s.v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        else:
            s.q, s.k, s.v = (_normal((B, T, h, D), dtype, g) for h in (Hq, Hkv, Hkv))
        s.dout = _normal((B, T, Hq, D), dtype, g) if case["train"] else None
        s.prefix = (1 + s.lengths // 4) if case["prefix"] else None
        s.slopes = _slopes(case) if case["slopes"] else None
    elif kind == "decode":
        Hq, Hkv = case["Hq"], case["Hkv"]
        if case["fused"]:                                        # keys and values of a slot side by side
            kv = _normal((B, T, 2, Hkv, D), dtype, g)
            s.k, s.v = kv[:, :, 0], kv[:, :, 1]
        else:
            s.k, s.v = (_normal((B, T, Hkv, D), dtype, g) for _ in range(2))
        s.q = _normal((s.n_seq, Hq, D), dtype, g)
        s.slopes = _slopes(case) if case["slopes"] else None
    elif kind in ("gated", "step"):
        s.x = _normal((B, T, D), dtype, g)
        # gates as a sigmoid leaves them, from forgetting at once to keeping for some hundred frames
        s.gate = torch.empty((B, T, D), device="cuda").normal_(2.0, 1.5, generator=g).sigmoid_().to(DTYPES[dtype])
        s.h0 = torch.empty((B, D), device="cuda").normal_(generator=g) if kind == "step" or case["state"] else None
        if kind == "step":
            s.reset, s.valid = torch.zeros((B, 1), dtype=torch.uint8, device="cuda"), torch.ones((B, 1), dtype=torch.uint8, device="cuda")
        else:
            s.dh = _normal((B, T, D), dtype, g)
            if case["state"]:                                    # a stream that goes on: no start at the first slot
                s.reset[:, 0] = 0
            s.dstate = torch.empty((B, D), device="cuda").normal_(generator=g) if case["state"] else None
    else:
        H = case["H"]
        if case["fused"]:                                        # the heads that are rotated, in front of those that are not
            s.x = _normal((B, T, H + 8, D), dtype, g)[:, :, :H]
        else:
            s.x = _normal((B, T, H, D), dtype, g)
        s.positions = torch.where(s.frame_idx >= 0, s.frame_idx + case["far"], s.frame_idx)
        s.frequencies = _frequencies(case)
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2310_10879_amd import bload
    c, kind = s.case, s.case["kind"]
    if kind == "attention":
        mask = bload.bload_segment_mask(s.reset, s.valid, causal=c["causal"], prefix=s.prefix, seq_id=s.seq_id)
        if not c["train"]:
            return [bload.bload_segment_attention(s.q, s.k, s.v, mask, cap=c["cap"], slopes=s.slopes)]
        out, saved = bload.bload_segment_attention(s.q, s.k, s.v, mask, cap=c["cap"], slopes=s.slopes, training=True)
        return [out, *bload.bload_segment_attention_backward(s.dout, s.q, s.k, s.v, out, saved, mask, cap=c["cap"],
                                                             slopes=s.slopes)]
    if kind == "decode":
        return [bload.bload_segment_attention_decode(s.q, s.k, s.v, s.block_of_seq, s.offset_of_seq, s.lengths,
                                                     cap=c["cap"], slopes=s.slopes)]
    if kind == "step":
        return list(bload.bload_gated_scan(s.gate, s.x, s.reset, s.valid, h0=s.h0))
    if kind == "gated":
        h, state = bload.bload_gated_scan(s.gate, s.x, s.reset, s.valid, h0=s.h0)
        dgate, dx, dh0 = bload.bload_gated_scan_backward(s.dh, s.gate, h, s.reset, s.valid, h0=s.h0, dstate=s.dstate)
        return [h, state, dgate, dx] + ([dh0] if c["state"] else [])
    return [bload.bload_rotary(s.x, s.positions, s.frequencies, layout=c["layout"], inverse=c["inverse"])]


def _run_plain(s):
    return {"attention": _plain_attention, "decode": _plain_decode, "gated": _plain_gated, "step": _plain_step,
            "rotary": _plain_rotary}[s.case["kind"]](s)


def _heads(x, Hq):
    """[B, T, H, D] -> float32 [B, Hq, T, D], shared heads repeated."""
    x = x.float().permute(0, 2, 1, 3)
    return x.repeat_interleave(Hq // x.shape[1], dim=1).contiguous()


def _plain_attention(s):
    c = s.case
    B, T, Hq, Hkv, D, dtype = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"], s.q.dtype
    same = (s.seq_id[:, :, None] == s.seq_id[:, None, :]) & (s.seq_id >= 0)[:, :, None]
    if c["causal"]:
        see = s.frame_idx[:, :, None] >= s.frame_idx[:, None, :]
        if s.prefix is not None:
            see = see | (s.frame_idx < s.prefix[s.seq_id.clamp(min=0).long()])[:, None, :]
        same = same & see
    hide = ~same[:, None]
    q, k, v = _heads(s.q, Hq), _heads(s.k, Hq), _heads(s.v, Hq)
    scale = 1.0 / math.sqrt(D)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    slope = None
    if c["cap"] > 0:
        p = torch.tanh(p / c["cap"])
        slope = 1.0 - p * p
        p = p * c["cap"]
    if s.slopes is not None:
        at = torch.arange(T, device="cuda")
        p = p - s.slopes[:, None, None] * (at[:, None] - at[None, :]).abs().float()
    p.masked_fill_(hide, -math.inf)
    p = torch.exp_(p - p.amax(dim=3, keepdim=True).clamp(min=-1e30))
    p /= p.sum(dim=3, keepdim=True).clamp(min=1e-30)             # a row that sees nothing stays 0
    out = torch.matmul(p, v)
    first = out.permute(0, 2, 1, 3).to(dtype).contiguous()
    if not c["train"]:
        return [first]
    do = _heads(s.dout, Hq)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds -= (do * out).sum(dim=3, keepdim=True)
    ds *= p
    del p
    ds *= scale
    if slope is not None:
        ds *= slope
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    dk, dv = (x.view(B, Hkv, Hq // Hkv, T, D).sum(dim=2) for x in (dk, dv))
    return [first] + [x.permute(0, 2, 1, 3).to(dtype).contiguous() for x in (dq, dk, dv)]


def _plain_decode(s):
    c = s.case
    n, T, Hq, Hkv, D = s.n_seq, c["T"], c["Hq"], c["Hkv"], c["D"]
    longest = int(min(T, _fill(c)[2].max()))
    at = torch.arange(longest, device="cuda")
    inside = at[None, :] < s.lengths[:, None]
    slot = (s.block_of_seq.long() * T + s.offset_of_seq.long())[:, None] + torch.where(inside, at[None, :], 0)
    k, v = (x.flatten(0, 1)[slot].float().permute(0, 2, 1, 3) for x in (s.k, s.v))           # [n, Hkv, L, D]
    q = s.q.float().view(n, Hkv, Hq // Hkv, D)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(D)                       # [n, Hkv, G, L]
    if c["cap"] > 0:
        p = torch.tanh(p / c["cap"]) * c["cap"]
    if s.slopes is not None:
        away = (s.lengths[:, None] - 1 - at[None, :]).float()
        p = p - s.slopes.view(1, Hkv, -1, 1) * away[:, None, None, :]
    p = p.masked_fill(~inside[:, None, None, :], -math.inf)
    p = torch.exp(p - p.amax(dim=3, keepdim=True))
    p = p / p.sum(dim=3, keepdim=True)
    return [torch.matmul(p, v.contiguous()).view(n, Hq, D).to(s.q.dtype)]


def _recurrence(a, x):
    """h[:, t] = a[:, t] * h[:, t - 1] + x[:, t] by doubling: after step d, h holds the part of the last 2 d frames."""
    d = 1
    while d < x.shape[1]:
        x = torch.cat([x[:, :d], x[:, d:] + a[:, d:] * x[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return x


def _carry(s):
    """1 where a slot goes on from the one in front of it (the first one: from the state handed in)."""
    on = (s.valid == 1) & (s.reset == 0)
    before = torch.cat([torch.full_like(s.valid[:, :1], s.h0 is not None), s.valid[:, :-1]], 1)
    return (on & (before == 1)).float()[:, :, None]


def _plain_forward(s):
    a = s.gate.float() * _carry(s)
    x = s.x.float() * s.valid.float()[:, :, None]
    if s.h0 is not None:
        x[:, 0] += a[:, 0] * s.h0
    return a, _recurrence(a, x)


def _plain_step(s):
    h = _plain_forward(s)[1]
    return [h.to(s.x.dtype), h[:, -1].contiguous()]


def _plain_gated(s):
    a, h = _plain_forward(s)
    dh = s.dh.float() * s.valid.float()[:, :, None]
    if s.dstate is not None:
        dh[:, -1] += s.dstate * s.valid[:, -1:].float()
    nxt = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    g = _recurrence(nxt.flip(1), dh.flip(1)).flip(1)
    before = torch.cat([torch.zeros_like(h[:, :1]) if s.h0 is None else s.h0[:, None], h[:, :-1]], 1)
    dgate = g * before * _carry(s)
    t = s.x.dtype
    return [h.to(t), h[:, -1].contiguous(), dgate.to(t), g.to(t)] + ([a[:, 0] * g[:, 0]] if s.case["state"] else [])


def _plain_rotary(s):
    c = s.case
    rot, x = c["rot"], s.x.float()
    angle = s.positions.double()[:, :, None, None] * s.frequencies.double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["inverse"]:
        sin = -sin
    if c["layout"] == "half":
        u, w = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([u * cos - w * sin, w * cos + u * sin, x[..., rot:]], 3)
    else:
        u, w = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.cat([torch.stack([u * cos - w * sin, w * cos + u * sin], 4).flatten(3), x[..., rot:]], 3)
    return [y.masked_fill_((s.positions < 0)[:, :, None, None], 0.0).to(s.x.dtype)]


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    B, T, D, kind, e = case["B"], case["T"], case["D"], case["kind"], BYTES[case["dtype"]]
    if kind == "step":
        return {"bytes": B * D * (3 * e + 8), "flops": 2 * B * D}
    length = _fill(case)[2].astype(np.float64)
    frames = float(length.sum())
    if kind == "attention":
        Hq, Hkv = case["Hq"], case["Hkv"]
        if case["prefix"]:
            head = 1 + length // 4                               # frames that all of the sequence sees
            pairs = float((length * (length + 1) / 2 + head * (head - 1) / 2).sum())
        else:
            pairs = float((length * (length + 1) / 2 if case["causal"] else length * length).sum())
        qo, kv = frames * Hq * D * e, frames * Hkv * D * e
        outs = B * T * Hq * D * e                                # padding is written too
        forward, flops = qo + 2 * kv + outs, 4 * D * Hq * pairs
        if not case["train"]:
            return {"bytes": forward + 2 * B * T, "flops": flops}
        return {"bytes": forward + 2 * B * T + qo + outs + 2 * B * T * Hkv * D * e, "flops": 3.5 * flops}
    if kind == "decode":
        Hq, Hkv, n = case["Hq"], case["Hkv"], len(length)
        return {"bytes": 2 * frames * Hkv * D * e + 2 * n * Hq * D * e + 12 * n, "flops": 4 * D * Hq * frames}
    if kind == "gated":
        state = 4 * B * D * (4 if case["state"] else 1)
        return {"bytes": e * D * (3 * frames + 3 * B * T) + 2 * B * T + state, "flops": 6 * frames * D}
    elements = B * T * case["H"] * D
    return {"bytes": e * (frames * case["H"] * D + elements) + 4 * B * T + 2 * case["rot"],
            "flops": 3 * frames * case["H"] * case["rot"]}


# ---------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "decode": _exact_decode, "gated": _exact_gated, "step": _exact_gated,
            "rotary": _exact_rotary}[case["kind"]](s)


def _visible(c, n, prefix):
    """[n, n]: may frame i of a sequence of n frames look at frame j."""
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None, :]
    see = torch.ones((n, n), dtype=torch.bool, device="cuda")
    if c["causal"]:
        see = j <= i
        if prefix is not None:
            see = see | (j < prefix)
    return see, (i - j).abs().double()


def _exact_attention(s):
    """Sequence by sequence, the gradients from torch's own differentiation."""
    c = s.case
    if s.n_seq > 3000:
        return None
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    grads = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (s.q, s.k, s.v)]
    block, first, length = (t.tolist() for t in (s.block_of_seq, s.offset_of_seq, s.lengths))
    prefix = s.prefix.tolist() if s.prefix is not None else [None] * s.n_seq
    for b, lo, n, pre in zip(block, first, length, prefix):
        at = (b, slice(lo, lo + n))
        q, k, v = (t[at].double().transpose(0, 1).contiguous().requires_grad_(c["train"]) for t in (s.q, s.k, s.v))
        see, away = _visible(c, n, pre)
        kk, vv = (t[:, None].expand(Hkv, Hq // Hkv, n, D).reshape(Hq, n, D) for t in (k, v))
        w = torch.bmm(q, kk.transpose(1, 2)) / math.sqrt(D)
        if c["cap"] > 0:
            w = c["cap"] * torch.tanh(w / c["cap"])
        if s.slopes is not None:
            w = w - s.slopes.double()[:, None, None] * away
        y = torch.bmm(torch.softmax(w.masked_fill(~see, -math.inf), dim=2), vv)
        out[at] = y.detach().transpose(0, 1)
        if c["train"]:
            y.backward(s.dout[at].double().transpose(0, 1))
            for to, t in zip(grads, (q, k, v)):
                to[at] = t.grad.transpose(0, 1)
    return [out] + (grads if c["train"] else [])


def _exact_decode(s):
    c = s.case
    if s.n_seq > 3000:
        return None
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    for i, (b, lo, n) in enumerate(zip(*(t.tolist() for t in (s.block_of_seq, s.offset_of_seq, s.lengths)))):
        k, v = (t[b, lo:lo + n].double().transpose(0, 1).contiguous() for t in (s.k, s.v))     # [Hkv, n, D]
        q = s.q[i].double().view(Hkv, Hq // Hkv, D)
        w = torch.bmm(k, q.transpose(1, 2)).transpose(1, 2) / math.sqrt(D)
        if c["cap"] > 0:
            w = c["cap"] * torch.tanh(w / c["cap"])
        if s.slopes is not None:
            w = w - s.slopes.double().view(Hkv, -1, 1) * torch.arange(n - 1, -1, -1, device="cuda").double()
        out[i] = torch.bmm(torch.softmax(w, dim=2), v).view(Hq, D)
    return [out]


def _exact_gated(s):
    """Frame by frame."""
    c, T = s.case, s.case["T"]
    B, D = c["B"], c["D"]
    h = torch.zeros((B, D), dtype=torch.float64, device="cuda") if s.h0 is None else s.h0.double()
    hs = torch.empty((B, T, D), dtype=torch.float64, device="cuda")
    goes_on = torch.zeros((B, T), dtype=torch.bool, device="cuda")
    alive = torch.full((B,), s.h0 is not None, device="cuda")
    first = h
    for t in range(T):
        valid = s.valid[:, t] == 1
        goes_on[:, t] = valid & (s.reset[:, t] == 0) & alive
        h = torch.where(goes_on[:, t, None], s.gate[:, t].double() * h, 0.0) + torch.where(valid[:, None], s.x[:, t].double(), 0.0)
        hs[:, t] = h
        alive = valid
    if c["kind"] == "step":
        return [hs, h]
    dgate, dx = torch.empty_like(hs), torch.empty_like(hs)
    g = torch.zeros((B, D), dtype=torch.float64, device="cuda") if s.dstate is None else s.dstate.double()
    for t in range(T - 1, -1, -1):
        g = torch.where((s.valid[:, t] == 1)[:, None], s.dh[:, t].double() + g, 0.0)
        dx[:, t] = g
        on = goes_on[:, t, None]
        dgate[:, t] = torch.where(on, g * (hs[:, t - 1] if t else first), 0.0)
        g = torch.where(on, g * s.gate[:, t].double(), 0.0)
    return [hs, h, dgate, dx] + ([g] if c["state"] else [])


def _exact_rotary(s):
    """A pair of elements is a complex number, times exp(i position frequency)."""
    c, x = s.case, s.x.double()
    rot = c["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       (-1.0 if c["inverse"] else 1.0) * s.positions.double()[:, :, None, None] * s.frequencies.double())
    y = torch.where((s.positions < 0)[:, :, None, None], 0.0, x)
    pairs = y[..., :rot]
    if c["layout"] == "half":
        z = torch.complex(*pairs.chunk(2, dim=3)) * turn
        y[..., :rot] = torch.cat([z.real, z.imag], 3)
    else:
        z = torch.complex(pairs[..., 0::2], pairs[..., 1::2]) * turn
        y[..., :rot] = torch.view_as_real(z).flatten(3)
    return [y]
