"""Element-wise bounds of the distillation's gradient: relative to q and p of the element, not to the row's largest.

In fp32 with u = 2^-24 (half a step), T the temperature, c2 = log2(e) / T:
  a = (z - m) c2            the difference, the quotient and the product are rounded, and so are the constant and T:   |a| 5 u
  a - l                     one rounding of at most |z - m| c2 + |l|, and l = log2(s):                                |a| u + 2 |l| u + the sum's relative error
  s                         `adds` additions on the longest way and, where a row is read again, as many rescalings, of exponentials off by an ulp (2 u) and by
                            their arguments: (2 adds + 2) u, and sum q |a| 5 u, which |a| of the element that counts bounds by the row's mean of q |a|
  exp2                      an ulp, 2 u, and ln 2 times the argument's error, below its error
  coef                      scale weight T and the product with it: 4 u
  m = lse T                 where the gradient is taken from lse: lse's own rounding, its product with T and the quotient's in lse: |lse| 4 u more in units of ln
The teacher's p alike with its k entries.  q - p is rounded once, and the result once to its type."""
import numpy as np

U32 = 2.0 ** -24


def parts(z, t, ids, temp):
    """q, the teacher's target (dense), |z - m| / T, lse / T's magnitude, in fp64; rows without entries have zeros."""
    rows, classes = z.shape
    x = z / temp
    m = x.max(1, keepdims=True)
    e = np.exp(x - m)
    s = e.sum(1, keepdims=True)
    q = e / s
    target, some, far = np.zeros_like(q), np.zeros(rows, bool), np.zeros(rows)
    for r in range(rows):
        there = (ids[r] >= 0) & (ids[r] < classes) & (t[r] > -np.inf)
        if there.any():
            v = t[r, there] / temp
            p = np.exp(v - v.max())
            np.add.at(target[r], ids[r, there], p / p.sum())
            some[r], far[r] = True, (v.max() - v).max()
    gap = np.where(np.isfinite(x), m - x, 0.0)
    return q * some[:, None], target, gap, far, np.abs(m + np.log(s)), some


def gradient(z, t, ids, weight, temp, scale, half_step, from_lse):
    """dz and its bound, element by element."""
    k = ids.shape[1]
    q, target, gap, far, lse, _ = parts(z, t, ids, temp)
    coef = (scale * temp * weight)[:, None]
    want = coef * (q - target)
    adds = 8 * 13 + z.shape[1] / 1024 + 40                          # of a thread, of a wave's tree and of the waves
    mean = (q * gap).sum(1, keepdims=True)
    log2e = 1.4427
    e_q = U32 * (6 * log2e * gap + 5 * log2e * mean + 2 * log2e * lse + 2 * adds + 16)
    if from_lse:
        e_q = e_q + U32 * 6 * lse
    e_p = U32 * (12 * log2e * far[:, None] + 2 * (k / 64 + 30) + 16)
    tiny = 2.0 ** -126                                              # results, and exponentials, below the least normal number may be 0
    return want, half_step * np.abs(want) + coef * ((e_q + U32) * q + (e_p + U32) * target + tiny) + tiny
