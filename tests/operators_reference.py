"""Plain 64-bit numpy forms of the operators on packed blocks, with bounds on what a kernel with
32-bit sums may be off.  ``u`` is half a step of the type: the largest relative error of one rounding."""
import numpy as np
import torch

U32 = 2.0 ** -24
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(TORCH[dtype]).eps / 2


def tiny(dtype):
    """Half the distance of subnormal numbers: the error of a rounding near 0."""
    return torch.finfo(TORCH[dtype]).smallest_normal * torch.finfo(TORCH[dtype]).eps / 2


def draw(rng, shape, dtype):
    """Unit normal values of the type, as a CPU tensor."""
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TORCH[dtype])


def wide(t):
    return t.detach().double().cpu().numpy()


def flags(rng, B, T, mean, p_pad=0.1):
    """Start table of B blocks of T slots: sequences of some ``mean`` frames, some followed by padding (padding may lie
    anywhere in a block, and a start flag may be missing behind it).  reset, valid, seq_id, n_seq."""
    reset, valid = np.zeros((B, T), np.uint8), np.zeros((B, T), np.uint8)
    seq_id = np.full((B, T), -1, np.int32)
    n = 0
    for b in range(B):
        t = 0
        while t < T:
            if rng.random() < p_pad:
                t += int(rng.integers(1, 4))
                continue
            e = min(T, t + int(rng.geometric(1.0 / mean)))
            valid[b, t:e] = 1
            seq_id[b, t:e] = n
            reset[b, t] = 1 if t > 0 and valid[b, t - 1] else rng.integers(0, 2)
            n += 1
            t = e
    return reset, valid, seq_id, n


def segments(reset, valid):
    """[(first, end)] of the sequences of one block."""
    out, T = [], len(valid)
    for t in range(T):
        if not valid[t]:
            continue
        if t == 0 or reset[t] or not valid[t - 1]:
            out.append([t, t + 1])
        else:
            out[-1][1] = t + 1
    return out


def visible(reset, valid, seq_id, causal, prefix):
    """bool[B, T, T]: does slot i's query see slot j's key."""
    B, T = valid.shape
    see = np.zeros((B, T, T), bool)
    for b in range(B):
        for f, e in segments(reset[b], valid[b]):
            for i in range(f, e):
                for_all = np.arange(f, e)
                if causal:
                    # (the table gives a prefix by the id at the slot in question: one id per sequence here)
                    p = 0 if prefix is None else max(0, int(prefix[seq_id[b, f]]))
                    for_all = for_all[(for_all <= i) | (for_all < f + p)]
                see[b, i, for_all] = True
    return see


def attention(q, k, v, see, scale, cap, slopes, dtype, dout=None):
    """Results and bounds of attention for float64 q [B, T, Hq, D], k and v [B, T, Hkv, D]: a dict of name -> (value, bound).

    With d_i the largest relative error that the 32-bit scores of row i leave on a probability, a computed p is off
    by (d_i + u) p, u from its rounding to the type; dp by D + 2 roundings; do.out by that of p in out."""
    B, T, Hq, D = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    u, z = half_step(dtype), tiny(dtype)
    names = ["out", "lse"] + (["dq", "dk", "dv"] if dout is not None else [])
    val = {n: np.zeros((B, Hq, T) if n == "lse" else (k.shape if n in ("dk", "dv") else q.shape)) for n in names}
    err = {n: np.zeros_like(val[n]) for n in names}
    val["lse"][:] = -np.inf
    at = np.arange(T)
    away = np.abs(at[:, None] - at[None, :])
    for b in range(B):
        rows = see[b].any(1)
        for h in range(Hq):
            Q, K, V = q[b, :, h], k[b, :, h // G], v[b, :, h // G]
            s = scale * Q @ K.T
            size = scale * np.abs(Q) @ np.abs(K).T
            keep = np.ones_like(s)
            s_err = (D + 4) * U32 * size
            if cap > 0:
                t = np.tanh(s / cap)
                s, keep = cap * t, 1 - t * t
                s_err = s_err + cap * 2.0 ** -21
            keep_err = 2 * s_err / cap + 2.0 ** -20 if cap > 0 else 0 * s
            if slopes is not None:
                s = s - slopes[h] * away
                s_err = s_err + 2 * U32 * np.abs(slopes[h] * away)
            s_err = s_err + 4 * U32 * (np.abs(s) + 1)
            m = np.where(see[b], s, -np.inf).max(1, keepdims=True, initial=-np.inf)
            m = np.where(np.isfinite(m), m, 0)
            p = np.where(see[b], np.exp(s - m), 0)
            total = p.sum(1, keepdims=True)
            p = p / np.where(total > 0, total, 1)
            d = np.where(see[b], s_err + 4 * U32 * np.abs(s - m), 0).max(1, keepdims=True)
            d = 2.5 * d + (T + 8) * U32                        # of p and of the sum that divides it
            out = p @ V
            out_err = (d + u) * (p @ np.abs(V)) + z * (see[b] @ np.abs(V))
            val["out"][b, :, h] = out
            err["out"][b, :, h] = out_err + u * np.abs(out) + z
            val["lse"][b, h, rows] = (np.log(np.where(total > 0, total, 1)) + m)[rows, 0]
            err["lse"][b, h, rows] = (d[:, 0] + 4 * U32 * (np.abs(val["lse"][b, h]) + 1))[rows]
            if dout is None:
                continue
            g = dout[b, :, h]
            # the backward pass takes p from the stored lse
            d = d + err["lse"][b, h][:, None] + 4 * U32 * np.where(rows, np.abs(np.where(rows, val["lse"][b, h], 0)), 0)[:, None]
            dp, dp_err = g @ V.T, (D + 2) * U32 * (np.abs(g) @ np.abs(V).T)
            delta = (g * out).sum(1, keepdims=True)
            delta_err = (np.abs(g) * (out_err + (2 * u * u + D * U32) * np.abs(out) + z)).sum(1, keepdims=True)
            x = (dp - delta) * keep
            ds = p * x
            ds_err = p * ((d + u) * np.abs(x) + dp_err + delta_err + keep_err * np.abs(dp - delta)) + z * see[b]
            val["dq"][b, :, h] = scale * ds @ K
            err["dq"][b, :, h] = scale * (ds_err + T * U32 * np.abs(ds)) @ np.abs(K)
            val["dk"][b, :, h // G] += scale * ds.T @ Q
            err["dk"][b, :, h // G] += scale * (ds_err + Hq * T * U32 * np.abs(ds)).T @ np.abs(Q)
            val["dv"][b, :, h // G] += p.T @ g
            err["dv"][b, :, h // G] += (p * (d + u + Hq * T * U32) + z * see[b]).T @ np.abs(g)
    for n in ("dq", "dk", "dv"):
        if n in val:
            err[n] += u * np.abs(val[n]) + z
    return {n: (val[n], err[n]) for n in names}


def gated(gate, x, reset, valid, h0, dtype, dout=None, dstate=None):
    """The recurrence and its gradients, frame by frame, with bounds.  k frames into a sequence a state has seen k
    roundings of products and sums, and as many of the maps that carry it from stretch to stretch."""
    B, T, D = x.shape
    u, z = half_step(dtype), tiny(dtype)
    h, size = np.zeros((B, T, D)), np.zeros((B, T, D))
    on = np.zeros((B, T), bool)
    age = np.zeros((B, T))
    at = np.zeros((B, D)) if h0 is None else h0.copy()
    big = np.abs(at)
    for t in range(T):
        live = valid[:, t] != 0
        before = np.full(B, h0 is not None) if t == 0 else valid[:, t - 1] != 0
        on[:, t] = live & (reset[:, t] == 0) & before
        a = np.where(on[:, t, None], gate[:, t], 0)
        at = np.where(live[:, None], a * at + x[:, t], 0)
        big = np.where(live[:, None], np.abs(a) * big + np.abs(x[:, t]), 0)
        age[:, t] = np.where(on[:, t], (age[:, t - 1] if t else 0) + 1, 1)
        h[:, t], size[:, t] = at, big
    state_err = (4 * age[..., None] + 16) * U32 * size
    out = {"h": (h, state_err + u * np.abs(h) + z), "state": (h[:, -1], state_err[:, -1])}
    if dout is None:
        return out
    g, gsize, left = np.zeros((B, T, D)), np.zeros((B, T, D)), np.zeros((B, T))
    at = np.zeros((B, D)) if dstate is None else dstate.copy()
    big = np.abs(at)
    for t in range(T - 1, -1, -1):
        live = (valid[:, t] != 0)[:, None]
        g[:, t] = np.where(live, dout[:, t] + at, 0)
        gsize[:, t] = np.where(live, np.abs(dout[:, t]) + big, 0)
        behind = on[:, t + 1] if t + 1 < T else np.zeros(B, bool)
        left[:, t] = np.where(behind, (left[:, t + 1] if t + 1 < T else 0) + 1, 1)
        a = np.where(on[:, t, None], gate[:, t], 0)
        at, big = a * g[:, t], np.abs(a) * gsize[:, t]
    g_err = (4 * left[..., None] + 16) * U32 * gsize
    first = np.zeros((B, 1, D)) if h0 is None else h0[:, None]
    prev = np.concatenate([first, h[:, :-1]], 1)
    prev_err = np.concatenate([0 * first, out["h"][1][:, :-1]], 1)        # the stored, rounded states
    dgate = np.where(on[..., None], g * prev, 0)
    out["dx"] = (g, g_err + u * np.abs(g) + z)
    out["dgate"] = (dgate, np.where(on[..., None], g_err * (np.abs(prev) + prev_err) + np.abs(g) * prev_err, 0) + (u + 2 * U32) * np.abs(dgate) + z)
    out["dh0"] = (at, (4 * left[:, 0, None] + 20) * U32 * big)
    return out


def rotary(x, positions, freq, layout, scale, inverse):
    """x: float64 [B, T, H, D]; freq: float64 [rot / 2].  The result and the sum of the sizes of its two terms."""
    rot = 2 * len(freq)
    y, size = x.copy(), np.abs(x)
    angle = positions[..., None, None].astype(np.float64) * freq
    c, s = scale * np.cos(angle), scale * np.sin(angle) * (-1 if inverse else 1)
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    size[..., lo] = size[..., hi] = abs(scale) * (np.abs(a) + np.abs(b))
    pad = positions < 0
    y[pad], size[pad] = 0, 0
    return y, size


def assert_close(got, want, bound, what):
    got = wide(got) if isinstance(got, torch.Tensor) else got
    same = np.isinf(want) & (got == want)
    off = np.where(same, 0, np.abs(got - np.where(same, 0, want)))
    bad = ~(off <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside the bound, first at {i}: got {got[i]} want {want[i]} "
                             f"bound {bound[i]}")
