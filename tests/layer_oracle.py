"""The linear layer, the gated projection and the distillation loss in fp64, written from their formulas, with bounds on what
rounding may do.  Rounding to a type is off by half a step, u = finfo.eps / 2 relative to the value."""
import math

import numpy as np
import torch
from scipy.special import erf

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]
# largest |act'| and |act''| of each, rounded up
SLOPE = {"none": 1.0, "relu": 1.0, "silu": 1.1, "gelu": 1.13, "gelu_tanh": 1.13}
CURVE = {"none": 0.0, "relu": 0.0, "silu": 0.5, "gelu": 0.8, "gelu_tanh": 0.8}


def f64(t):
    return t.detach().cpu().double().numpy()


def act(name, v):
    """(act(v), act'(v))"""
    if name == "none":
        return v, np.ones_like(v)
    if name == "relu":
        return np.maximum(v, 0), (v > 0).astype(float)
    if name == "silu":
        s = 1 / (1 + np.exp(-v))
        return v * s, s * (1 + v * (1 - s))
    if name == "gelu":
        cdf = 0.5 * (1 + erf(v / math.sqrt(2)))
        return v * cdf, cdf + v * np.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    t = np.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)


def sums(a, b, terms):
    """a @ b, and how far fp32 sums of `terms` products in any order may be off: each partial sum is rounded once."""
    return a @ b, (terms + 4) * U[torch.float32] * (np.abs(a) @ np.abs(b))


# The functions of one variable: exponential and reciprocal instructions are off by an ulp each, their arguments by one rounding of a value of
# magnitude below 12 where the result matters, erf of the device library by a few ulps.  16 roundings of 32 bits relative to |v| + 1 cover them.
def act_err(v):
    return 16 * U[torch.float32] * (np.abs(v) + 1)


def linear_fwd(name, x, w, bias, res, dtype):
    """y, pre and the bounds of both."""
    pre, e_pre = sums(x, w, x.shape[1])
    if bias is not None:
        pre = pre + bias
        e_pre = e_pre + U[torch.float32] * np.abs(pre)
    y, _ = act(name, pre)
    e = SLOPE[name] * e_pre + (act_err(pre) if name != "none" else 0)
    if res is not None:
        y = y + res
        e = e + U[torch.float32] * np.abs(y)
    return y, pre, U[dtype] * np.abs(y) + e, U[dtype] * np.abs(pre) + e_pre


def products_bwd(dzs, x, ws, e_dzs, dtype, wdtype):
    """dx = sum dz w^T, dw = x^T dz for gradients known up to e_dz: values and bounds."""
    dx = e_dx = 0
    dws = []
    for dz, w, e in zip(dzs, ws, e_dzs):
        d, ed = sums(dz, w.T, dz.shape[1] * len(dzs))
        dx, e_dx = dx + d, e_dx + ed + e @ np.abs(w.T)
        d, ed = sums(x.T, dz, x.shape[0])
        dws.append((d, U[wdtype] * np.abs(d) + ed + np.abs(x.T) @ e))
    return dx, U[dtype] * np.abs(dx) + e_dx, dws


def linear_bwd(name, dy, x, w, pre, dtype, wdtype):
    slope = act(name, pre)[1] if name != "none" else np.ones_like(dy)
    dz = dy * slope
    fine = 0 if name == "none" else np.abs(dy) * act_err(pre)       # dz in fp32
    e_dz = np.zeros_like(dz) if name == "none" else U[dtype] * np.abs(dz) + fine
    dx, e_dx, [(dw, e_dw)] = products_bwd([dz], x, [w], [e_dz], dtype, wdtype)
    db = dz.sum(0)
    e_db = (dz.shape[0] + 4) * U[torch.float32] * np.abs(dz).sum(0) + (fine.sum(0) if name != "none" else 0)
    return dx, e_dx, dw, e_dw, db, e_db


def gated_fwd(name, x, wg, wu, dtype):
    g, e_g = sums(x, wg, x.shape[1])
    u, e_u = sums(x, wu, x.shape[1])
    a, _ = act(name, g)
    h = a * u
    e = (SLOPE[name] * e_g + act_err(g)) * np.abs(u) + (np.abs(a) + e_g) * e_u + U[torch.float32] * np.abs(h)
    return h, g, u, U[dtype] * np.abs(h) + e, U[dtype] * np.abs(g) + e_g, U[dtype] * np.abs(u) + e_u


def gated_bwd(name, dh, x, wg, wu, g, u, dtype, wdtype):
    """g, u: as kept (storage type), or None: computed again."""
    e_g = e_u = 0
    if g is None:
        g, e_g = sums(x, wg, x.shape[1])
        u, e_u = sums(x, wu, x.shape[1])
    a, s = act(name, g)
    dg, du = dh * u * s, dh * a
    e_dg = U[dtype] * np.abs(dg) + np.abs(dh) * ((np.abs(u) + e_u) * (act_err(g) + CURVE[name] * e_g) + SLOPE[name] * e_u) + 2 * U[torch.float32] * np.abs(dg)
    e_du = U[dtype] * np.abs(du) + np.abs(dh) * (act_err(g) + SLOPE[name] * e_g) + U[torch.float32] * np.abs(du)
    return products_bwd([dg, du], x, [wg, wu], [e_dg, e_du], dtype, wdtype)


def distill(z, t, ids, weight, temp, scale):
    """loss, row losses, lse, dz; each row by the definition."""
    rows, classes = z.shape
    row_loss, lse, dz = np.zeros(rows), np.zeros(rows), np.zeros(z.shape)
    for r in range(rows):
        s = z[r] / temp
        high = s.max()
        lse[r] = high + math.log(np.exp(s - high).sum()) if high > -math.inf else -math.inf
        q = np.exp(s - lse[r]) if high > -math.inf else np.zeros(classes)
        there = [j for j in range(ids.shape[1]) if 0 <= ids[r, j] < classes and t[r, j] > -math.inf]
        if not there:
            continue
        v = t[r, there] / temp
        p = np.exp(v - v.max())
        p /= p.sum()
        target = np.zeros(classes)
        for j, pj in zip(there, p):
            target[ids[r, j]] += pj
            if pj > 0:
                row_loss[r] += pj * (math.log(pj) - (s[ids[r, j]] - lse[r])) if s[ids[r, j]] > -math.inf else math.inf
        row_loss[r] *= temp * temp
        if weight[r] != 0:
            dz[r] = scale * weight[r] * temp * (q - target)
    loss = scale * sum(w * l for w, l in zip(weight, row_loss) if w != 0)
    return loss, row_loss, lse, dz
