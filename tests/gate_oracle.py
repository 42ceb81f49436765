"""The gated recurrence in fp64 with bounds that hold for gates near their ends: what is kept and what is taken in are each off relative to themselves, however small.  u = finfo.eps / 2."""
import numpy as np
import torch

from layer_oracle import U, act, act_err
from sequence_oracle import sigmoid

U32 = U[torch.float32]
TINY = 2.0 ** -125


def recur(x, g, o, act_name, borders, h0, dy, dlast, dtype):
    """{name: (value, bound)}.

    With e = exp(-|g|), the smaller of a and 1 - a is e / (1 + e): |g| log2(e) is off by the constant's 0.3 u and the product's u, which is 1.3 |g| u of e; exponential and reciprocal by an ulp,
    2 u, each, the sum and the product by u: (1.3 |g| + 6) u of the smaller one, and below 2^-126 it may be flushed to 0.  The larger one is 1 minus that: it has the smaller one's error and u.
    A position makes a h + (1 - a) x of h: beside the errors of a and 1 - a, a product and a sum are rounded, and a is a factor of the spans' products, each rounded too, whose compositions add two
    roundings for every two positions at least, and as many for the spans of spans: 8 u of a |h| + (1 - a) |x| cover them.  Later positions scale errors by their a.  Backwards alike."""
    a, rest = sigmoid(g), sigmoid(-g)
    k = (1.3 * np.abs(g) + 6) * U32 * np.minimum(a, rest) + TINY    # of a, and of 1 - a
    val, slope = (np.ones_like(x), np.zeros_like(x)) if o is None else act(act_name, o)
    e_act = np.zeros_like(x) if o is None else act_err(o)
    h, before, e_h, e_before, m_before, dh, m_dh, e_dh = (np.full(x.shape, np.nan) for _ in range(8))
    last, e_last, dh0, e_dh0 = h0.copy(), np.zeros_like(h0), dlast.copy(), np.zeros_like(dlast)
    used = np.zeros(len(x), bool)
    for s, (b, e) in enumerate(borders):
        now, err, most = h0[s].copy(), np.zeros(x.shape[1]), np.abs(h0[s])
        for t in range(b, e):
            used[t] = True
            before[t], e_before[t], m_before[t] = now, err, most
            now, new = a[t] * now + rest[t] * x[t], a[t] * most + rest[t] * np.abs(x[t])
            err = a[t] * err + k[t] * (most + np.abs(x[t])) + 8 * U32 * new
            most = new
            h[t], e_h[t] = now, err
        last[s], e_last[s] = now, err
        d = dy * val
        e_d = np.abs(dy) * e_act + U32 * np.abs(d)
        r, err, most = dlast[s].copy(), np.zeros(x.shape[1]), np.abs(dlast[s])
        for t in range(e - 1, b - 1, -1):
            dh[t], m_dh[t] = d[t] + r, np.abs(d[t]) + most
            e_dh[t] = e_d[t] + err + U32 * m_dh[t]
            r, err, most = a[t] * dh[t], a[t] * e_dh[t] + (k[t] + 8 * U32 * a[t]) * m_dh[t], a[t] * m_dh[t]
        dh0[s], e_dh0[s] = r, err
    y, dx, apart = h * val, rest * dh, np.abs(before) + np.abs(x)
    dg, do = dh * (before - x) * a * rest, dy * h * slope
    e_y = e_h * np.abs(val) + (np.abs(h) + e_h) * e_act + U32 * np.abs(y)
    e_dx = rest * e_dh + (k + U32 * rest) * m_dh
    # dh (before - x) a (1 - a): each factor's error, and three products
    e_dg = a * rest * (e_dh * (apart + e_before) + m_dh * (e_before + U32 * apart)) + (k + 4 * U32 * a * rest) * m_dh * (apart + e_before)
    e_do = np.abs(dy) * (e_h * np.abs(slope) + (np.abs(h) + e_h) * e_act) + 2 * U32 * np.abs(do)
    out = {n: (v, U[dtype] * np.abs(v) + e) for n, v, e in (("y", y, e_y), ("dx", dx, e_dx), ("dg", dg, e_dg), ("do", do, e_do))}
    out.update(last=(last, e_last + U32 * np.abs(last)), dh0=(dh0, e_dh0 + U32 * np.abs(dh0)), used=used)
    return out
