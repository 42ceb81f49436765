"""Group normalisation on the GPU against fp64: tokens, images and volumes, one position and one channel, groups across vectors, odd sizes and pitches, both types, gradients, means far
from zero, streams and graphs."""
import numpy as np
import pytest

import sequence_oracle as S
from layer_oracle import f64

pytestmark = pytest.mark.gpu

# n, s, c, groups, act, affine, dtype, pad
CASES = [(1, 1, 1, 1, "none", True, "fp32", 0), (3, 1, 8, 8, "silu", True, "bf16", 0), (7, 1, 96, 3, "gelu", True, "fp32", 3), (300, 1, 512, 4, "none", True, "bf16", 0),
         (65, 1, 1000, 8, "silu", False, "bf16", 8), (17, 1, 4096, 32, "none", True, "bf16", 0), (5, 1, 8192, 1, "gelu_tanh", True, "bf16", 0), (9, 1, 2044, 7, "relu", True, "fp32", 0),
         (33, 1, 2050, 2, "silu", True, "bf16", 1), (2, 1, 40000, 5, "none", True, "bf16", 0), (4, 49, 64, 8, "relu", True, "bf16", 0), (2, 63, 30, 10, "silu", True, "fp32", 2),
         (3, 196, 256, 32, "silu", True, "bf16", 0), (1, 4097, 24, 3, "gelu", True, "bf16", 8), (2, 3000, 6, 2, "none", False, "fp32", 0), (1, 70000, 16, 4, "relu", True, "bf16", 0),
         (5, 2, 300, 1, "gelu_tanh", True, "bf16", 0), (1, 100, 1028, 257, "silu", True, "bf16", 4), (40, 5, 128, 2, "none", True, "fp32", 0), (1, 9000, 1, 1, "none", True, "fp32", 0),
         # tokens whose rows are all of a group, of no power of two of vectors; groups and rows that are not of whole vectors; images of few positions
         (700, 1, 192, 1, "gelu", True, "bf16", 0), (33, 1, 440, 1, "silu", True, "fp32", 1), (1500, 1, 576, 16, "gelu", True, "bf16", 0), (90, 1, 1001, 7, "silu", True, "fp32", 3),
         (21, 1, 4100, 41, "relu", False, "bf16", 0), (19, 1, 8190, 2, "gelu_tanh", True, "bf16", 2), (5, 1, 7000, 7000, "none", True, "bf16", 0), (3000, 1, 12, 4, "silu", True, "fp32", 0),
         (50, 2, 1024, 32, "silu", True, "bf16", 0), (33, 3, 64, 8, "relu", True, "fp32", 0), (9, 7, 8, 1, "none", True, "bf16", 0), (6, 30, 2048, 2, "gelu", True, "bf16", 8),
         # parts of groups in several waves, a thread's vectors of one group, more rows than work-groups
         (700, 1, 4096, 1, "silu", True, "bf16", 0), (40, 1, 6000, 1, "none", True, "fp32", 0), (33, 1, 8192, 2, "relu", True, "bf16", 0), (12, 1, 16384, 1, "gelu", True, "bf16", 0),
         (9, 1, 12000, 3, "silu", True, "fp32", 0), (9000, 1, 64, 2, "silu", True, "bf16", 0), (2600, 1, 2048, 1, "none", False, "bf16", 0), (50, 1, 1000, 5, "gelu", True, "fp32", 0)]


def ptr(t):
    return None if t is None else t.data_ptr()


def make(torch, seed, n, s, c, affine, dtype, pad, mean=0.0):
    gen = torch.Generator().manual_seed(seed)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32

    def mat(shift):
        t = torch.full((n * s, c + pad), float("nan"))
        t[:, :c] = torch.randn(n * s, c, generator=gen) + shift
        return t.to(kind).cuda()[:, :c]
    d = dict(x=mat(mean + torch.randn(c, generator=gen)), dy=mat(0.0), kind=kind)
    d["gamma"], d["beta"] = ((torch.randn(c, generator=gen) * 0.3 + 1).cuda(), (torch.randn(c, generator=gen) * 0.3).cuda()) if affine else (None, None)
    return d


def call(torch, L, d, n, s, c, groups, act, pad, eps=1e-5):
    A = L.abi
    acts = {"none": A.ACT_NONE, "relu": A.ACT_RELU, "silu": A.ACT_SILU, "gelu": A.ACT_GELU, "gelu_tanh": A.ACT_GELU_TANH}
    st = torch.cuda.current_stream().cuda_stream
    desc = L.group_norm_desc(n, s, c, groups, act=acts[act], dtype=A.BF16 if d["kind"] == torch.bfloat16 else A.F32, eps=eps, ldx=c + pad, ldy=c + pad)
    ws = torch.full((max(L.group_norm_workspace_bytes(desc, w) for w in (A.GROUP_NORM_FWD, A.GROUP_NORM_BWD)) + 16,), 255, dtype=torch.uint8, device="cuda")
    out = {k: torch.full((n * s, c + pad), 777.0, dtype=d["kind"], device="cuda") for k in ("y", "dx")}
    out["mean"], out["rstd"] = (torch.full((n, groups), 777.0, device="cuda") for _ in range(2))
    out["dgamma"], out["dbeta"] = (torch.full((c,), 777.0, device="cuda") for _ in range(2))
    L.group_norm_fwd(desc, ptr(d["x"]), ptr(d["gamma"]), ptr(d["beta"]), ptr(out["y"]), ptr(out["mean"]), ptr(out["rstd"]), ptr(ws), st)
    ws.fill_(255)
    L.group_norm_bwd(desc, ptr(d["dy"]), ptr(d["x"]), ptr(d["gamma"]), ptr(d["beta"]), ptr(out["mean"]), ptr(out["rstd"]), ptr(out["dx"]), ptr(out["dgamma"]), ptr(out["dbeta"]),
                    ptr(ws), st)
    return out


def within(name, got, want):
    off = np.abs(f64(got) - want[0])
    assert (off <= want[1]).all(), (name, np.argwhere(~(off <= want[1]))[0], off.max())


def check(d, out, n, s, c, groups, act, eps=1e-5):
    gamma = np.ones(c) if d["gamma"] is None else f64(d["gamma"])
    beta = np.zeros(c) if d["beta"] is None else f64(d["beta"])
    x = f64(d["x"])
    y, mean, rstd = S.group_norm_fwd(x, n, s, groups, gamma, beta, act, eps, d["kind"])
    within("mean", out["mean"], mean)
    within("rstd", out["rstd"], rstd)
    within("y", out["y"][:, :c], y)
    dx, dg, db = S.group_norm_bwd(f64(d["dy"]), x, n, s, groups, gamma, beta, f64(out["mean"]), f64(out["rstd"]), act, d["kind"])
    within("dx", out["dx"][:, :c], dx)
    within("dgamma", out["dgamma"], dg)
    within("dbeta", out["dbeta"], db)
    for k in ("y", "dx"):
        assert bool((out[k][:, c:] == out[k].new_tensor(777.0)).all()), k          # nothing between the rows


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_fp64(i):
    import torch
    import paper_1807_02037_amd as L
    n, s, c, groups, act, affine, dtype, pad = CASES[i]
    d = make(torch, i, n, s, c, affine, dtype, pad)
    out = call(torch, L, d, n, s, c, groups, act, pad)
    torch.cuda.synchronize()
    check(d, out, n, s, c, groups, act)
    again = call(torch, L, d, n, s, c, groups, act, pad)
    torch.cuda.synchronize()
    for k, v in out.items():
        assert torch.equal(v, again[k]), k


def test_gradients_against_differences():
    rng = np.random.default_rng(3)
    import torch
    n, s, c, groups, eps = 2, 3, 6, 2, 1e-5
    x, dy = rng.standard_normal((n * s, c)), rng.standard_normal((n * s, c))
    gamma, beta = rng.standard_normal(c), rng.standard_normal(c)

    def loss():
        return (S.group_norm_fwd(x, n, s, groups, gamma, beta, "silu", eps, torch.float32)[0][0] * dy).sum()
    _, mean, rstd = S.group_norm_fwd(x, n, s, groups, gamma, beta, "silu", eps, torch.float32)
    want = S.group_norm_bwd(dy, x, n, s, groups, gamma, beta, mean[0], rstd[0], "silu", torch.float32)
    for t, (v, _) in zip((x, gamma, beta), want):
        for i in np.ndindex(t.shape):
            t0, step = t[i], 1e-5
            t[i] = t0 + step
            up = loss()
            t[i] = t0 - step
            down = loss()
            t[i] = t0
            assert abs((up - down) / (2 * step) - v[i]) < 1e-6, i


@pytest.mark.parametrize("n,s,c,groups", [(3, 1, 512, 2), (2, 50, 64, 4), (1, 5000, 32, 2)])
def test_means_far_from_zero(n, s, c, groups):
    """Deviations of 1 around 3000 in 32 bits, whose squares' differences would hold nothing; and values all alike, whose variance is 0."""
    import torch
    import paper_1807_02037_amd as L
    d = make(torch, 7, n, s, c, True, "fp32", 0, mean=3000.0)
    out = call(torch, L, d, n, s, c, groups, "none", 0)
    torch.cuda.synchronize()
    check(d, out, n, s, c, groups, "none")
    d["x"].fill_(3001.5)
    out = call(torch, L, d, n, s, c, groups, "none", 0, eps=1e-3)
    torch.cuda.synchronize()
    assert bool((out["mean"] == 3001.5).all()) and torch.equal(out["y"], d["beta"].expand(n * s, c))
    check(d, out, n, s, c, groups, "none", eps=1e-3)


def test_a_sample_keeps_its_nan_to_itself():
    import torch
    import paper_1807_02037_amd as L
    for n, s in ((5, 1), (5, 70)):
        d = make(torch, 4, n, s, 64, True, "bf16", 0)
        clean = call(torch, L, d, n, s, 64, 4, "silu", 0)
        d["x"][2 * s, 20] = float("nan")                           # sample 2, group 1
        got = call(torch, L, d, n, s, 64, 4, "silu", 0)
        torch.cuda.synchronize()
        for k in ("y", "dx"):
            a, b = got[k].reshape(n, s, 4, 16), clean[k].reshape(n, s, 4, 16)
            assert a[2, :, 1].isnan().all()
            a[2, :, 1], b[2, :, 1] = 0, 0
            assert torch.equal(a, b)


def test_optional_outputs_and_no_samples():
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    for n, s in ((6, 1), (2, 33)):
        d = make(torch, 2, n, s, 40, True, "bf16", 0)
        full = call(torch, L, d, n, s, 40, 5, "silu", 0)
        desc = L.group_norm_desc(n, s, 40, 5, act=A.ACT_SILU)
        ws = torch.empty(max(L.group_norm_workspace_bytes(desc, w) for w in (0, 1)) + 16, dtype=torch.uint8, device="cuda")
        st, y = torch.cuda.current_stream().cuda_stream, torch.empty_like(full["y"])
        L.group_norm_fwd(desc, ptr(d["x"]), ptr(d["gamma"]), ptr(d["beta"]), ptr(y), None, None, ptr(ws), st)
        assert torch.equal(y, full["y"])
        args = [desc] + [ptr(t) for t in (d["dy"], d["x"], d["gamma"], d["beta"], full["mean"], full["rstd"])]
        for names in (("dx",), ("dgamma",), ("dbeta",), ("dgamma", "dbeta")):
            got = {k: torch.empty_like(full[k]) for k in names}
            L.group_norm_bwd(*args, ptr(got.get("dx")), ptr(got.get("dgamma")), ptr(got.get("dbeta")), ptr(ws), st)
            for k in names:
                assert torch.equal(got[k], full[k]), k
    empty, dg, db = L.group_norm_desc(0, 5, 40, 5), torch.full((40,), 7.0, device="cuda"), torch.full((40,), 7.0, device="cuda")
    L.group_norm_fwd(empty, None, None, None, None, None, None, None, st)
    L.group_norm_bwd(empty, None, None, None, None, None, None, None, ptr(dg), ptr(db), None, st)
    torch.cuda.synchronize()
    assert not dg.any() and not db.any()


def test_many_samples_in_parts():
    """More than is taken at a time; the oracle on a few samples."""
    import torch
    import paper_1807_02037_amd as L
    n, s, c, groups = 90, 1600, 512, 8
    d = make(torch, 9, n, s, c, True, "bf16", 0)
    out = call(torch, L, d, n, s, c, groups, "relu", 0)
    torch.cuda.synchronize()
    for i in (0, 44, 89):
        part = dict(d, x=d["x"][i * s:(i + 1) * s], dy=d["dy"][i * s:(i + 1) * s])
        one = call(torch, L, part, 1, s, c, groups, "relu", 0)
        got = {k: out[k][i * s:(i + 1) * s] if k in ("y", "dx") else out[k][i:i + 1] for k in ("y", "dx", "mean", "rstd")}
        check(part, dict(got, dgamma=one["dgamma"], dbeta=one["dbeta"]), 1, s, c, groups, "relu")


def test_streams_and_graphs():
    import torch
    import paper_1807_02037_amd as L
    shapes = [(6, 300, 64, 8), (50, 1, 256, 4)]
    ds = [make(torch, i, n, s, c, True, "bf16", 0) for i, (n, s, c, _) in enumerate(shapes)]
    eager = [call(torch, L, d, *sh, "silu", 0) for d, sh in zip(ds, shapes)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for d, sh in zip(ds, shapes):
        with torch.cuda.stream(side):
            call(torch, L, d, *sh, "silu", 0)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(call(torch, L, d, *sh, "silu", 0))
            graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        call(torch, L, ds[0], *shapes[0], "silu", 0)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            for k in a:
                assert torch.equal(a[k], b[k]), k
                a[k].fill_(777.0)
        torch.cuda.synchronize()
