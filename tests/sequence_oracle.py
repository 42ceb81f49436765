"""The gated recurrence, group normalisation, the 8-bit linear layer and the verification of drafts in fp64 (whole numbers where they are), written from their formulas, with bounds on
what rounding may do.  Rounding to a type is off by half a step, u = finfo.eps / 2 relative to the value."""
import numpy as np
import torch

from layer_oracle import U, act, act_err

U32 = U[torch.float32]
CUT = 2.0 ** -99


def sigmoid(v):
    return np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))


def spans(rows, seqs, offsets):
    if offsets is None:
        each = rows // seqs
        return [(s * each, (s + 1) * each) for s in range(seqs)]
    return [(int(offsets[s]), int(offsets[s + 1])) for s in range(seqs)]


def recur(x, g, o, act_name, borders, h0, dy=None, dlast=None, dtype=torch.bfloat16):
    """{name: (value, bound)}.  A position takes h to a h + (1 - a) x: in fp32 a is off by (|g| + 4) u relative to itself and the sums by u of what they add, which are no larger than
    |h| and |x|; later positions scale these errors by their a.  Spans composed in another order than one position after the other round the same products, once more for each
    composition: (8 + |g|) u of all that goes in at each position covers both.  Far gates: the exponential is cut at 2^100, so a is off by 2^-100 at most where it is smaller, and 1 - a below
    2^-126 may be flushed to 0: CUT = 2^-99 of what they are multiplied with, however small the result (e^-200 is no number of 32 bits)."""
    rows, c = x.shape
    a, rest = sigmoid(g), sigmoid(-g)
    k = (8 + np.abs(g)) * U32
    val, slope = (np.ones_like(x), np.zeros_like(x)) if o is None else act(act_name, o)
    e_act = np.zeros_like(x) if o is None else act_err(o)
    h, before, e_h, e_before, m_before = (np.full(x.shape, np.nan) for _ in range(5))
    last, e_last = h0.copy(), np.zeros_like(h0)
    used = np.zeros(rows, bool)
    for s, (b, e) in enumerate(borders):
        now, err, most = h0[s].copy(), np.zeros(c), np.abs(h0[s])
        for t in range(b, e):
            used[t] = True
            before[t], e_before[t], m_before[t] = now, err, most
            now = a[t] * now + rest[t] * x[t]
            new = a[t] * most + rest[t] * np.abs(x[t])
            err = a[t] * err + k[t] * (new + most + np.abs(x[t])) + CUT * most
            most = new
            h[t], e_h[t] = now, err
        last[s], e_last[s] = now, err
    y = h * val
    out = {"y": (y, U[dtype] * np.abs(y) + e_h * np.abs(val) + (np.abs(h) + e_h) * e_act + U32 * np.abs(y)), "last": (last, e_last + U32 * np.abs(last)), "used": used}
    if dy is None:
        return out
    e = dy * val
    e_e = np.abs(dy) * e_act + U32 * np.abs(e)
    dh, e_dh, m_dh = (np.full(x.shape, np.nan) for _ in range(3))
    dh0, e_dh0 = dlast.copy(), np.zeros_like(dlast)
    for s, (b, en) in enumerate(borders):
        r, err, most = dlast[s].copy(), np.zeros(c), np.abs(dlast[s])
        for t in range(en - 1, b - 1, -1):
            dh[t], m_dh[t] = e[t] + r, np.abs(e[t]) + most
            e_dh[t] = e_e[t] + err + U32 * m_dh[t]
            r, err, most = a[t] * dh[t], a[t] * e_dh[t] + (k[t] * a[t] + CUT) * m_dh[t], a[t] * m_dh[t]
        dh0[s], e_dh0[s] = r, err
    dx, dg, do = rest * dh, dh * (before - x) * a * rest, dy * h * slope
    apart = np.abs(before) + np.abs(x)
    e_dx = rest * e_dh + (k * rest + CUT) * m_dh
    e_dg = a * rest * (e_dh * (np.abs(before - x) + e_before) + m_dh * (e_before + U32 * apart)) + (2 * k * a * rest + 2 * CUT) * m_dh * (apart + e_before)
    e_do = np.abs(dy) * (e_h * np.abs(slope) + (np.abs(h) + e_h) * (e_act if o is not None else 0)) + 2 * U32 * np.abs(do)
    for name, v, b in (("dx", dx, e_dx), ("dg", dg, e_dg), ("do", do, e_do)):
        out[name] = (v, U[dtype] * np.abs(v) + b)
    out["dh0"] = (dh0, e_dh0 + U32 * np.abs(dh0))
    return out


def _grouped(t, n, s, groups):
    return t.reshape(n, s, groups, -1)


def norm_terms(n, s, cg):
    """Roundings that follow one another in a sum over a group at most: rows of a thread, threads of a column, chunks and channels by 256 threads, the tree."""
    return 24 + min(s, 560 + s / 512) + s * cg / 4096


def group_norm_fwd(x, n, s, groups, gamma, beta, act_name, eps, dtype):
    """y, mean, rstd and their bounds.  Means are joined from rows and channels: each join rounds values no larger than the largest |x| (with K joins, K u of it), and deviations are off by
    as much; in the variance that error meets a deviation, or itself."""
    v = _grouped(x, n, s, groups)
    ax = (1, 3)
    k = 3 * norm_terms(n, s, v.shape[3]) * U32
    mean, var = v.mean(ax, keepdims=True), v.var(ax, keepdims=True)
    most = np.abs(v).max(ax, keepdims=True)
    e_mean = k * most
    e_var = 2 * k * (var + np.sqrt(var) * most) + e_mean ** 2
    rstd = 1 / np.sqrt(var + eps)
    e_rstd = rstd * (np.minimum(1, 0.5 * e_var / (var + eps) * (1 + e_var / (var + eps))) + 6 * U32)
    y, e_y = _norm_out(v, mean, rstd, e_mean, e_rstd, gamma, beta, act_name)[:2]
    y = y.reshape(x.shape)
    return (y, e_y.reshape(x.shape) + U[dtype] * np.abs(y)), (mean.reshape(n, groups), e_mean.reshape(n, groups)), (rstd.reshape(n, groups), e_rstd.reshape(n, groups))


def _norm_out(v, mean, rstd, e_mean, e_rstd, gamma, beta, act_name):
    from layer_oracle import SLOPE
    groups = v.shape[2]
    ga, be = gamma.reshape(groups, -1), beta.reshape(groups, -1)
    hat = (v - mean) * rstd
    e_hat = rstd * (e_mean + U32 * (np.abs(v) + np.abs(mean))) + np.abs(v - mean) * e_rstd + 3 * U32 * np.abs(hat)
    pre = ga * hat + be
    e_pre = np.abs(ga) * e_hat + 3 * U32 * (np.abs(pre) + np.abs(be))
    y, slope = act(act_name, pre)
    return y, SLOPE[act_name] * e_pre + (act_err(pre) if act_name not in ("none", "relu") else 0), hat, e_hat, pre, e_pre, slope


def group_norm_bwd(dy, x, n, s, groups, gamma, beta, mean, rstd, act_name, dtype):
    """dx, dgamma, dbeta and their bounds; mean and rstd as given."""
    from layer_oracle import CURVE
    v, d = _grouped(x, n, s, groups), _grouped(dy, n, s, groups)
    mean, rstd, ga = mean.reshape(n, 1, groups, 1), rstd.reshape(n, 1, groups, 1), gamma.reshape(groups, -1)
    _, _, hat, e_hat, pre, e_pre, slope = _norm_out(v, mean, rstd, 0, 0, gamma, beta, act_name)
    e_slope = CURVE[act_name] * e_pre + (act_err(pre) if act_name not in ("none", "relu") else 0)
    if act_name == "relu":
        e_slope = (np.abs(pre) <= e_pre) * 1.0                     # either side of the border
    dv = d * slope
    e_dv = np.abs(d) * e_slope + U32 * np.abs(dv)
    k = (norm_terms(n, s, v.shape[3]) + n) * U32
    ax = (1, 3)
    u, w = ga * dv, ga * dv * hat
    m1, m2 = u.mean(ax, keepdims=True), w.mean(ax, keepdims=True)
    e_w = np.abs(ga) * (e_dv * np.abs(hat) + np.abs(dv) * e_hat)
    e_m1 = (np.abs(ga) * e_dv).mean(ax, keepdims=True) + k * np.abs(u).mean(ax, keepdims=True)
    e_m2 = e_w.mean(ax, keepdims=True) + k * np.abs(w).mean(ax, keepdims=True)
    dx = rstd * (u - m1 - hat * m2)
    e_dx = rstd * (np.abs(ga) * e_dv + e_m1 + np.abs(hat) * e_m2 + np.abs(m2) * e_hat + 4 * U32 * (np.abs(u) + np.abs(m1) + np.abs(hat * m2)))
    dx, e_dx = dx.reshape(x.shape), e_dx.reshape(x.shape)
    db, dg = dv.sum((0, 1)).ravel(), (dv * hat).sum((0, 1)).ravel()
    e_db = (e_dv + k * np.abs(dv)).sum((0, 1)).ravel()
    e_dg = (e_dv * np.abs(hat) + np.abs(dv) * e_hat + k * np.abs(dv * hat)).sum((0, 1)).ravel()
    return (dx, e_dx + U[dtype] * np.abs(dx)), (dg, e_dg + U32 * np.abs(dg)), (db, e_db + U32 * np.abs(db))
