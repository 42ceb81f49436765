"""Group normalisation of more samples than a grid of the three launches takes (2^22 work-groups, two of them for each group's sums): several launches one after the other, every sample against fp64, and
the sums for gamma and beta over all of them."""
import numpy as np
import pytest

import sequence_oracle as S
import test_gpu_group_norm as N
from layer_oracle import U, f64

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


def launches(torch, call, name):
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    return sum(e.count for e in prof.key_averages() if name in e.key)


# samples, positions, channels, groups, act, dtype, parts: 2^22 / (2 groups) samples in each
@pytest.mark.parametrize("n,s,c,groups,act,dtype,parts", [(1500001, 2, 3, 3, "none", "fp32", 3), (800000, 2, 6, 6, "silu", "bf16", 3), (2 ** 21 + 5, 2, 4, 1, "relu", "bf16", 2)])
def test_samples_in_several_launches(n, s, c, groups, act, dtype, parts):
    import torch
    import paper_1807_02037_amd as L
    d = N.make(torch, 3, n, s, c, True, dtype, 0)
    d["dy"].mul_(0.2).add_(1).add_(d["x"])                         # gradients that go with x: the sums grow with the samples, so that a lost part shows
    out = N.call(torch, L, d, n, s, c, groups, act, 0)
    torch.cuda.synchronize()
    x, dy, gamma, beta = (f64(d[k]) for k in ("x", "dy", "gamma", "beta"))
    y, mean, rstd = S.group_norm_fwd(x, n, s, groups, gamma, beta, act, 1e-5, d["kind"])
    N.within("mean", out["mean"], mean)
    N.within("rstd", out["rstd"], rstd)
    N.within("y", out["y"], y)
    dx, _, _ = S.group_norm_bwd(dy, x, n, s, groups, gamma, beta, f64(out["mean"]), f64(out["rstd"]), act, d["kind"])
    # means of a group's few values; the bound of a sum over n samples is not theirs
    small = S.group_norm_bwd(dy[:s], x[:s], 1, s, groups, gamma, beta, f64(out["mean"])[:1], f64(out["rstd"])[:1], act, d["kind"])[0]
    N.within("dx of the first sample", out["dx"][:s], small)
    assert (np.abs(f64(out["dx"]) - dx[0]) <= dx[1]).all()
    # a thread of 32 adds up every 32nd sample, eight at a time: n / 256 sums one after the other, a tree of three, 32 threads, and what a sample's positions and the functions round
    m, r = (np.repeat(f64(out[k]), c // groups, 1)[:, None, :] for k in ("mean", "rstd"))
    hat = (x.reshape(n, s, c) - m) * r
    pre = gamma * hat + beta
    dv = dy.reshape(n, s, c) * S.act(act, pre)[1]
    k = (n / 256 + 3 + 32 + 8 + 64) * U32
    # silu's slope is off by act_err, at most 16 u (|v| + 1); relu's at its border by 1 for values within rounding of it
    fuzzy = np.abs(dy.reshape(n, s, c)) * (S.act_err(pre) if act == "silu" else (np.abs(pre) <= 8 * U32 * (np.abs(gamma * hat) + np.abs(beta))) if act == "relu" else 0)
    for name, terms, scale in (("dgamma", dv * hat, np.abs(hat)), ("dbeta", dv, 1.0)):
        want, most = terms.sum((0, 1)), np.abs(terms).sum((0, 1))
        bound = k * most + (fuzzy * scale).sum((0, 1))
        assert (np.abs(f64(out[name]) - want) <= bound).all(), (name, np.abs(f64(out[name]) - want) / bound)
        if act != "relu":
            assert (bound < np.abs(terms[:2 ** 22 // (2 * groups)].sum((0, 1))) / 4).all() and (bound < np.abs(terms[-(n // 4):].sum((0, 1))) / 4).all(), name      # a part that is lost would be seen
    assert launches(torch, lambda: N.call(torch, L, d, n, s, c, groups, act, 0), "norm_stats") == parts
    assert launches(torch, lambda: N.call(torch, L, d, n, s, c, groups, act, 0), "norm_dx") == parts
