"""Plain 64-bit numpy forms of the norms, the short convolution and the selective scan on packed blocks, with bounds on what a
kernel of 32-bit arithmetic may be off.  Every function gives a dict of name -> (value, bound).  U32 is one rounding in 32 bits; the
bounds are first-order sums of the roundings on the way, carried along with the values."""
import numpy as np

from operators_reference import U32, half_step, tiny


def rounded(value, error, dtype):
    return value, error + half_step(dtype) * (np.abs(value) + error) + tiny(dtype)


def sigmoid(x):
    return np.exp(-np.logaddexp(0, -x))


def sigmoid_off(x):
    """Relative: the argument of the exponential is rounded twice, 1.5 |x| U32 each (its result's part of 1 + e^-x is below 1), the
    exponential, the sum and the reciprocal to a unit or two."""
    return (3 * np.abs(x) + 8) * U32


def goes_on(reset, valid, has_state):
    before = np.concatenate([np.full((len(valid), 1), bool(has_state)), valid[:, :-1] != 0], 1)
    return (valid != 0) & (reset == 0) & before


# ---------------------------------------------------------------- norms


def norm(s, weight, bias, live, eps, center, dtype, dout=None, dsum=None):
    """s: float64 [rows, D], what is normalised; live: bool[rows]; dout, dsum like s (dsum may be None)."""
    rows, D = s.shape
    # a sum over a row: up to 64 + D / 256 additions in a lane, ten between lanes and wavefronts
    n = (90 + D / 256) * U32
    # a column's: rows / 1024 in a lane, then lanes, wavefronts and up to 64 + 16 parts
    m = (100 + rows / 1024) * U32
    w = np.ones(D) if weight is None else weight
    b = np.zeros(D) if bias is None else bias
    s = np.where(live[:, None], s, 0)
    mean = s.mean(1, keepdims=True) if center else np.zeros((rows, 1))
    mean_off = (n * np.abs(s).mean(1, keepdims=True) + 2 * U32 * np.abs(mean)) if center else 0 * mean
    d = s - mean
    d_off = mean_off + U32 * np.abs(d)
    var = (d * d).mean(1, keepdims=True)
    var_off = (2 * np.abs(d) * d_off + d_off ** 2).mean(1, keepdims=True) + (n + 4 * U32) * var
    r = 1 / np.sqrt(var + eps) if eps > 0 else np.where(var > 0, 1 / np.sqrt(np.where(var > 0, var, 1)), 0)
    # (relative; once a variance is lost in its error, the bound says nothing)
    rho = var_off / (2 * np.maximum(var + eps - var_off, 1e-300)) + 4 * U32
    u = d * r
    u_off = r * d_off * (1 + rho) + np.abs(u) * (rho + 2 * U32)
    y = u * w + b
    y_off = np.abs(w) * u_off + U32 * (2 * np.abs(u * w) + np.abs(y))
    off = lambda x: np.where(live[:, None], x, 0)
    out = {"out": tuple(off(x) for x in rounded(y, y_off, dtype)), "mean": (mean, mean_off),
           "r": (np.where(live[:, None], r, 0), np.where(live[:, None], r * rho, 0))}
    if dout is None:
        return out
    dy = np.where(live[:, None], dout, 0)
    g = dy * w
    c1 = g.mean(1, keepdims=True) if center else np.zeros((rows, 1))
    c1_off = (n + 2 * U32) * np.abs(g).mean(1, keepdims=True) if center else 0 * c1
    c2 = (g * u).mean(1, keepdims=True)
    c2_off = (n + 4 * U32) * np.abs(g * u).mean(1, keepdims=True) + (np.abs(g) * u_off).mean(1, keepdims=True)
    inner = g - c1 - u * c2
    inner_off = c1_off + np.abs(u) * c2_off + u_off * np.abs(c2) + 4 * U32 * (np.abs(g) + np.abs(c1) + np.abs(u * c2))
    dx = r * inner + (0 if dsum is None else dsum)
    dx_off = r * inner_off + np.abs(r * inner) * (rho + U32) + U32 * np.abs(dx)
    out["dx"] = tuple(off(x) for x in rounded(dx, dx_off, dtype))
    out["dweight"] = (dy * u).sum(0), (np.abs(dy) * u_off).sum(0) + m * np.abs(dy * u).sum(0) + tiny("f32")
    out["dbias"] = dy.sum(0), m * np.abs(dy).sum(0) + tiny("f32")
    return out


# ---------------------------------------------------------------- short convolution


def conv(x, weight, bias, reset, valid, silu, state, dtype, dout=None, dstate=None):
    """x: float64 [B, T, D]; weight [D, K]; state [B, K - 1, D] or None."""
    B, T, D = x.shape
    K = weight.shape[1]
    live, on = valid != 0, goes_on(reset, valid, state is not None)
    front = np.zeros((B, K - 1, D)) if state is None else state
    rows = np.concatenate([front, x], 1)
    on = np.concatenate([np.ones((B, K - 1), bool), on], 1)                # of the rows
    see = np.zeros((K, B, T), bool)                                        # tap j of slot t
    for t in range(T):
        reach = live[:, t].copy()
        for j in range(K):
            see[j, :, t] = reach
            reach &= on[:, K - 1 + t - j]
    keep = np.zeros((K - 1, B), bool)                                      # row i of the state behind
    reach = live[:, -1].copy()
    for i in range(K - 2, -1, -1):
        keep[i] = reach
        reach &= on[:, T + i]
    taps = [np.where(see[j][..., None], rows[:, K - 1 - j:K - 1 - j + T], 0) for j in range(K)]
    b = np.zeros(D) if bias is None else bias
    p = np.where(live[..., None], b + sum(weight[:, K - 1 - j] * taps[j] for j in range(K)), 0)
    p_off = (K + 2) * U32 * (np.abs(b) + sum(np.abs(weight[:, K - 1 - j] * taps[j]) for j in range(K)))
    sg = sigmoid(p)
    y, y_off = (p * sg, 1.1 * p_off + np.abs(p * sg) * (sigmoid_off(p) + U32)) if silu else (p, p_off)
    cut = lambda pair: tuple(np.where(live[..., None], v, 0) for v in pair)
    left = np.stack([np.where(keep[i][:, None], rows[:, T + i], 0) for i in range(K - 1)], 1) if K > 1 else np.zeros((B, 0, D))
    out = {"out": cut(rounded(y, y_off, dtype)), "state": (left, np.zeros_like(left))}
    if dout is None:
        return out
    dp = np.where(live[..., None], dout, 0)
    dp_off = np.zeros_like(dp)
    if silu:
        slope = sg * (1 + p * (1 - sg))
        # the slope moves by half of what p is off at most; its own arithmetic: sigmoid twice, a product, a sum
        slope_off = 0.5 * p_off + sg * (1 + np.abs(p)) * (2 * sigmoid_off(p) + 6 * U32)
        dp, dp_off = dp * slope, np.abs(dp) * (slope_off + U32 * np.abs(slope))
    d, d_off, size = (np.zeros_like(rows) for _ in range(3))
    dw, dw_off = np.zeros_like(weight), np.zeros_like(weight)
    for j in range(K):
        w, at = weight[:, K - 1 - j], slice(K - 1 - j, K - 1 - j + T)
        mine = see[j][..., None]
        d[:, at] += np.where(mine, w * dp, 0)
        d_off[:, at] += np.where(mine, np.abs(w) * dp_off, 0)
        size[:, at] += np.where(mine, np.abs(w * dp), 0)
        dw[:, K - 1 - j] = (dp * taps[j]).sum((0, 1))
        # 64 slots and more in a lane, runs and wavefronts, the parts
        dw_off[:, K - 1 - j] = (dp_off * np.abs(taps[j])).sum((0, 1)) + 200 * U32 * np.abs(dp * taps[j]).sum((0, 1)) + tiny("f32")
    if dstate is not None:
        for i in range(K - 1):
            d[:, T + i] += np.where(keep[i][:, None], dstate[:, i], 0)
            size[:, T + i] += np.where(keep[i][:, None], np.abs(dstate[:, i]), 0)
    d, d_off = rounded(d, d_off + (K + 2) * U32 * size, dtype)
    none = ~live[..., None]
    out["dx"] = np.where(none, 0, d[:, K - 1:]), np.where(none, 0, d_off[:, K - 1:])
    out["dstate_in"] = d[:, :K - 1], d_off[:, :K - 1]
    out["dweight"] = dw, dw_off
    out["dbias"] = dp.sum((0, 1)), dp_off.sum((0, 1)) + 200 * U32 * np.abs(dp).sum((0, 1)) + tiny("f32")
    return out


# ---------------------------------------------------------------- selective scan


def scan(x, dt, rate, b, c, reset, valid, skip, z, dt_bias, softplus, h0, dtype, dout=None, dstate=None):
    """x, dt, z: float64 [B, T, D]; rate [D, N]; b, c [B, T, G, N]; h0, dstate [B, D, N]."""
    B, T, D = x.shape
    G, N = b.shape[2:]
    live, on = (valid != 0)[..., None], goes_on(reset, valid, h0 is not None)
    none = np.zeros(D)
    skip, has_z = none if skip is None else skip, z is not None
    v = np.where(live, dt + (none if dt_bias is None else dt_bias), 0)
    x = np.where(live, x, 0)
    step = np.logaddexp(v, 0) if softplus else v
    step = np.where(live, step, 0)
    v_off = U32 * np.where(live, np.abs(dt) + np.abs(none if dt_bias is None else dt_bias), 0)
    slope = sigmoid(v) if softplus else np.ones_like(v)
    # softplus: the exponential of |v| to (1.5 |v| + 2) of a rounding, twelve more roundings behind it
    step_off = slope * (v_off + U32 * np.abs(v)) + (step * (2 * np.abs(v) + 16) * U32 if softplus else U32 * np.abs(step))
    to_d = lambda t: np.where(live[:, :, None], t, 0).repeat(D // G, 2)     # [B, T, G, N] -> [B, T, D, N]
    bb, cc = to_d(b), to_d(c)
    a = np.exp(step[..., None] * rate)
    # the exponential's argument is a product of rounded factors; joined chunks add as many roundings again
    a_off = 2 * (np.abs(rate) * step_off[..., None] + 3 * U32 * np.abs(step[..., None] * rate) + 3 * U32)
    a, a_off = (np.where(on[..., None, None], t, 0) for t in (a, a_off))
    ux = step * x
    ux_off = np.abs(x) * step_off + U32 * np.abs(ux)
    u = ux[..., None] * bb
    u_off = ux_off[..., None] * np.abs(bb) + 2 * U32 * np.abs(u)
    h, h_off = np.zeros((B, T + 1, D, N)), np.zeros((B, T + 1, D, N))
    h[:, 0] = 0 if h0 is None else h0
    for t in range(T):
        moved = a[:, t] * h[:, t]
        h[:, t + 1] = moved + u[:, t]
        h_off[:, t + 1] = a[:, t] * h_off[:, t] + np.abs(moved) * (a_off[:, t] + 4 * U32) + u_off[:, t] + 4 * U32 * np.abs(u[:, t])
    hs, hs_off = h[:, 1:], h_off[:, 1:]
    y = (cc * hs).sum(3) + skip * x
    y_off = (np.abs(cc) * hs_off).sum(3) + (N + 6) * U32 * (np.abs(cc * hs).sum(3) + np.abs(skip * x))
    zz = np.where(live, z, 0) if has_z else None
    sg = sigmoid(zz) if has_z else 1
    gate, gate_off = (zz * sg, np.abs(zz * sg) * (sigmoid_off(zz) + 2 * U32)) if has_z else (1.0, 0.0)
    res, res_off = y * gate, y_off * np.abs(gate) + np.abs(y) * gate_off
    cut = lambda pair: tuple(np.where(live, t, 0) for t in pair)
    out = {"out": cut(rounded(res, res_off, dtype)), "state": (h[:, -1], h_off[:, -1])}
    if dout is None:
        return out
    do = np.where(live, dout, 0)
    dy, dy_off = do * gate, np.abs(do) * (gate_off + U32 * np.abs(gate))
    g, g_off, back, back_off = (np.zeros((B, T, D, N)) for _ in range(4))
    at = np.zeros((B, D, N)) if dstate is None else np.where(live[:, -1, :, None], dstate, 0)
    at_off = np.zeros_like(at)
    for t in range(T - 1, -1, -1):
        own = dy[:, t, :, None] * cc[:, t]
        g[:, t] = own + at
        g_off[:, t] = at_off + dy_off[:, t, :, None] * np.abs(cc[:, t]) + 2 * U32 * (np.abs(own) + np.abs(at))
        at = a[:, t] * g[:, t]
        at_off = a[:, t] * g_off[:, t] + np.abs(at) * (a_off[:, t] + 4 * U32)
        back[:, t], back_off[:, t] = at, at_off
    per = lambda t: t.reshape(B, T, G, D // G, N).sum(3)
    dc, db = dy[..., None] * hs, ux[..., None] * g
    out["dc"] = rounded(per(dc), per(np.abs(dy[..., None]) * hs_off + dy_off[..., None] * np.abs(hs) + (D + 20) * U32 * np.abs(dc)), dtype)
    out["db"] = rounded(per(db), per(np.abs(ux[..., None]) * g_off + ux_off[..., None] * np.abs(g) + (D + 20) * U32 * np.abs(db)), dtype)
    q, q_off = (g * bb).sum(3), (g_off * np.abs(bb) + (N + 6) * U32 * np.abs(g * bb)).sum(3)
    front, front_off = h[:, :-1], h_off[:, :-1]
    k = back * front
    k_off = back_off * np.abs(front) + np.abs(back) * front_off + U32 * np.abs(k)
    w, w_off = (k * rate).sum(3), (k_off * np.abs(rate) + (N + 8) * U32 * np.abs(k * rate)).sum(3)
    dx = step * q + skip * dy
    dx_off = step_off * np.abs(q) + np.abs(step) * q_off + np.abs(skip) * dy_off + 4 * U32 * (np.abs(step * q) + np.abs(skip * dy))
    out["dx"] = cut(rounded(dx, dx_off, dtype))
    ds = w + x * q
    ds_off = w_off + np.abs(x) * q_off + 3 * U32 * (np.abs(w) + np.abs(x * q))
    dv, dv_off = ds * slope, ds_off * slope + np.abs(ds) * slope * (sigmoid_off(v) + np.abs(v_off) + U32)
    out["ddt"] = cut(rounded(dv, dv_off, dtype))
    n = (B * T + 100) * U32                                                # additions of a sum over all slots, at most
    out["drate"] = (k * step[..., None]).sum((0, 1)), \
        (k_off * np.abs(step[..., None]) + np.abs(k) * step_off[..., None] + n * np.abs(k * step[..., None])).sum((0, 1)) + tiny("f32")
    dv, dv_off = cut((dv, dv_off))
    out["ddt_bias"] = dv.sum((0, 1)), (dv_off + n * np.abs(dv)).sum((0, 1)) + tiny("f32")
    out["dskip"] = (dy * x).sum((0, 1)), (dy_off * np.abs(x) + n * np.abs(dy * x)).sum((0, 1)) + tiny("f32")
    if has_z:
        s = sg * (1 + zz * (1 - sg))
        s_off = sg * (1 + np.abs(zz)) * (2 * sigmoid_off(zz) + 6 * U32)
        out["dz"] = cut(rounded(do * y * s, np.abs(do) * (y_off * np.abs(s) + np.abs(y) * s_off + 3 * U32 * np.abs(y * s)), dtype))
    out["dh0"] = at, at_off
    return out
