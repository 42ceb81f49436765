"""The linear layer in 8-bit integers on the GPU: steps and sums exact, outputs against fp64; sizes of every tile, split and join, odd ones and pitches, both types, ties, zeros, the ends of
the types, values that are not finite, graphs."""
import numpy as np
import pytest

from layer_oracle import SLOPE, U, act, act_err, f64

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24

# m, k, n, act, bias, res, dtype, pad
CASES = [(1, 1, 1, "none", False, False, "fp32", 0), (1, 16, 8, "silu", True, True, "bf16", 0), (3, 17, 5, "gelu", True, False, "fp32", 1), (1, 4096, 4096, "none", True, True, "bf16", 0),
         (2, 1000, 2050, "silu", True, True, "bf16", 3), (5, 4097, 33, "relu", False, True, "fp32", 0), (8, 2048, 8192, "gelu", True, False, "bf16", 0),
         (24, 2048, 4096, "gelu_tanh", True, True, "bf16", 8), (33, 520, 776, "none", True, False, "fp32", 0), (64, 8190, 256, "none", False, False, "bf16", 0),
         (100, 700, 1000, "silu", True, True, "fp32", 5), (300, 1024, 1024, "gelu", True, True, "bf16", 0), (1000, 64, 100, "none", False, False, "bf16", 0),
         (1030, 1032, 1100, "relu", True, True, "bf16", 8), (513, 2064, 4104, "none", True, True, "fp32", 0), (4100, 528, 2056, "silu", True, True, "bf16", 0),
         (16, 40000, 70, "none", False, False, "fp32", 0), (2, 131072, 16, "none", False, False, "fp32", 0),
         # up to 64 rows in one round: blocks of 16 and of 32 columns, lines and stages that end inside, one short row of weights; and what takes the tiles beside them
         (3, 1, 1, "none", True, True, "bf16", 0), (32, 144, 4096, "silu", True, True, "bf16", 4), (17, 2064, 4097, "gelu", True, True, "fp32", 3), (32, 2032, 8190, "none", False, True, "bf16", 2),
         (33, 3000, 4096, "relu", True, False, "fp32", 0), (64, 8192, 50, "none", True, True, "bf16", 6), (63, 530, 8192, "gelu_tanh", True, True, "bf16", 0), (40, 127, 5001, "none", False, False, "fp32", 1),
         (7, 12288, 37, "none", True, True, "bf16", 0), (9, 12300, 300, "none", True, False, "bf16", 0), (24, 2048, 8200, "gelu", True, True, "bf16", 0), (65, 2560, 500, "silu", True, True, "bf16", 0)]


def ptr(t):
    return None if t is None else t.data_ptr()


def steps(x):
    """Steps and scales of rows: 127 x / most in fp64 is within 2^-52 of the quotient, which is a tie or 2^-34 from one.  Rows that are not finite: no steps, NaN."""
    finite = np.isfinite(x).all(1, keepdims=True)
    x = np.where(finite, x, 0)
    most = np.where(finite, np.abs(x).max(1, keepdims=True), np.nan)
    return np.rint(127 * x / np.where(most > 0, most, 1)), (most / 127).astype(np.float32).astype(float)[:, 0]


def make(torch, seed, m, k, n, bias, res, dtype, pad):
    gen = torch.Generator().manual_seed(seed)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32

    def mat(rows, cols, extra, scale=1.0):
        t = torch.full((rows, cols + extra), float("nan"))
        t[:, :cols] = torch.randn(rows, cols, generator=gen) * scale
        return t.to(kind).cuda()[:, :cols]
    return dict(x=mat(m, k, pad), w=mat(k, n, pad, k ** -0.5), bias=torch.randn(n, generator=gen).cuda() if bias else None, res=mat(m, n, pad) if res else None, kind=kind)


def setup(torch, L, d, m, k, n, name, pad):
    A = L.abi
    acts = {"none": A.ACT_NONE, "relu": A.ACT_RELU, "silu": A.ACT_SILU, "gelu": A.ACT_GELU, "gelu_tanh": A.ACT_GELU_TANH}
    desc = L.linear_q8_desc(m, n, k, act=acts[name], dtype=A.BF16 if d["kind"] == torch.bfloat16 else A.F32, ldx=k + pad, ldw=n + pad, ldy=n + pad, ldr=n + pad)
    wq = torch.full((L.linear_q8_weight_bytes(desc),), 85, dtype=torch.int8, device="cuda")
    sw = torch.full((n,), 777.0, device="cuda")
    ws = torch.full((L.linear_q8_workspace_bytes(desc) + 16,), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    L.linear_q8_weight(desc, ptr(d["w"]), ptr(wq), ptr(sw), s)
    return desc, wq, sw, ws, s


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_fp64(i):
    import torch
    import paper_1807_02037_amd as L
    m, k, n, name, bias, res, dtype, pad = CASES[i]
    d = make(torch, i, m, k, n, bias, res, dtype, pad)
    desc, wq, sw, ws, s = setup(torch, L, d, m, k, n, name, pad)
    kp = wq.numel() // n
    y = torch.full((m, n + pad), 777.0, dtype=d["kind"], device="cuda")
    L.linear_q8_fwd(desc, ptr(d["x"]), ptr(wq), ptr(sw), ptr(d["bias"]), ptr(d["res"]), ptr(y), ptr(ws), s)
    xq, sx = torch.full((m, kp), 85, dtype=torch.int8, device="cuda"), torch.full((m,), 777.0, device="cuda")
    L.linear_q8_rows(desc, ptr(d["x"]), ptr(xq), ptr(sx), s)
    both = torch.full_like(y, 777.0)
    L.linear_q8_product(desc, ptr(xq), ptr(sx), ptr(wq), ptr(sw), ptr(d["bias"]), ptr(d["res"]), ptr(both), ptr(ws), s)
    torch.cuda.synchronize()
    assert torch.equal(y, both)
    want_x, want_sx = steps(f64(d["x"]))
    want_w, want_sw = steps(f64(d["w"]).T)
    got_w = wq.reshape(n, kp).cpu().numpy()
    assert (xq.cpu().numpy()[:, :k] == want_x).all() and not xq[:, k:].any()
    assert (got_w[:, :k] == want_w).all() and not got_w[:, k:].any()
    assert np.array_equal(f64(sx), want_sx) and np.array_equal(f64(sw), want_sw)
    pre = (want_x @ want_w.T) * want_sx[:, None] * want_sw         # fp64 holds the sums
    e = 4 * U32 * np.abs(pre)
    if bias:
        pre = pre + f64(d["bias"])
        e = e + U32 * np.abs(pre)
    want = act(name, pre)[0]
    e = SLOPE[name] * e + (act_err(pre) if name != "none" else 0)
    if res:
        want = want + f64(d["res"])
        e = e + U32 * np.abs(want)
    off, allowed = np.abs(f64(y[:, :n]) - want), e + U[d["kind"]] * np.abs(want)
    assert (off <= allowed).all(), (np.argwhere(~(off <= allowed))[0], off.max())
    assert bool((y[:, n:] == y.new_tensor(777.0)).all())
    if res:                                                        # over the residual
        L.linear_q8_fwd(desc, ptr(d["x"]), ptr(wq), ptr(sw), ptr(d["bias"]), ptr(d["res"]), ptr(d["res"]), ptr(ws), s)
        torch.cuda.synchronize()
        assert torch.equal(d["res"], y[:, :n])


def test_largest_sums():
    """All steps 127: the largest sums that a row gives, over splits too."""
    import torch
    import paper_1807_02037_amd as L
    for m, k, n in ((1, 131072, 24), (40, 131072, 40), (300, 100000, 16)):
        d = dict(x=torch.ones(m, k, device="cuda"), w=torch.ones(k, n, device="cuda"), kind=torch.float32)
        d["w"][:, 1::2] = -1
        desc, wq, sw, ws, s = setup(torch, L, d, m, k, n, "none", 0)
        y = torch.empty(m, n, device="cuda")
        L.linear_q8_fwd(desc, ptr(d["x"]), ptr(wq), ptr(sw), None, None, ptr(y), ptr(ws), s)
        torch.cuda.synchronize()
        want = k * 127.0 ** 2 * float(np.float32(1 / 127)) ** 2
        off = np.abs(np.abs(f64(y)) - want)
        assert (off <= 4 * U32 * want).all() and (f64(y)[:, 1::2] < 0).all() and (f64(y)[:, ::2] > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steps_at_their_borders(dtype):
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    k = 64
    half = torch.arange(k) - 31.5                                  # ties where the largest is 127
    # the seventh row's spacing is beyond fp32: what linspace makes of it is not finite
    rows = [torch.cat([half[:-1], torch.tensor([127.0])]), torch.cat([half[:-1], torch.tensor([-127.0])]) * 2.0 ** 100, torch.cat([half[:-1], torch.tensor([127.0])]) * 2.0 ** -130,
            torch.zeros(k), torch.full((k,), -0.0), torch.full((k,), 3.3e38), torch.linspace(-3.3e38, 3.3e38, k), torch.full((k,), 2.0 ** -133),
            torch.linspace(-1, 1, k), torch.linspace(0, 1e-30, k)]
    x = torch.stack(rows).to(kind).cuda()
    m = len(rows)
    desc = L.linear_q8_desc(m, 1, k, dtype=A.BF16 if dtype == "bf16" else A.F32)
    xq, sx = torch.full((m, k), 85, dtype=torch.int8, device="cuda"), torch.full((m,), 777.0, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    L.linear_q8_rows(desc, ptr(x), ptr(xq), ptr(sx), s)
    torch.cuda.synchronize()
    want, scale = steps(f64(x))
    assert (xq.cpu().numpy() == want).all(), np.argwhere(xq.cpu().numpy() != want)
    assert np.allclose(f64(sx), scale, rtol=2.0 ** -23, atol=2.0 ** -148, equal_nan=True)
    for bad in (float("nan"), float("inf"), float("-inf")):
        z = x.clone()
        z[2, 17] = bad
        L.linear_q8_rows(desc, ptr(z), ptr(xq), ptr(sx), s)
        torch.cuda.synchronize()
        assert sx[2].isnan() and not xq[2].any() and not sx[[0, 1, 3, 4, 5]].isnan().any()
    # a column that is not finite, a row of zeros: their own results alone
    d = make(torch, 1, 20, 100, 40, False, False, dtype, 0)
    d["w"][3, 7], d["x"][5] = float("inf"), 0.0
    desc, wq, sw, ws, s = setup(torch, L, d, 20, 100, 40, "none", 0)
    y = torch.empty(20, 40, dtype=kind, device="cuda")
    L.linear_q8_fwd(desc, ptr(d["x"]), ptr(wq), ptr(sw), None, None, ptr(y), ptr(ws), s)
    torch.cuda.synchronize()
    assert y[:, 7].isnan().all() and not y[:, :7].isnan().any() and not y[:, 8:].isnan().any() and not y[5, 8:].any()


def test_streams_and_graphs():
    import torch
    import paper_1807_02037_amd as L
    shapes = [(1, 4096, 1024), (40, 1024, 512)]
    ds = [make(torch, i, m, k, n, True, True, "bf16", 0) for i, (m, k, n) in enumerate(shapes)]
    kept = [setup(torch, L, d, *sh, "silu", 0) for d, sh in zip(ds, shapes)]

    def call(i, out, ws):
        d, (desc, wq, sw, _, _) = ds[i], kept[i]
        L.linear_q8_fwd(desc, ptr(d["x"]), ptr(wq), ptr(sw), ptr(d["bias"]), ptr(d["res"]), ptr(out), ptr(ws), torch.cuda.current_stream().cuda_stream)
    eager = [torch.empty_like(d["res"]) for d in ds]
    for i in (0, 1):
        call(i, eager[i], kept[i][3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], [torch.empty_like(d["res"]) for d in ds]
    spaces = [torch.empty_like(k[3]) for k in kept]
    for i in (0, 1):
        with torch.cuda.stream(side):
            call(i, outs[i], spaces[i])
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call(i, outs[i], spaces[i])
            graphs.append(g)
    again = torch.empty_like(eager[0])
    for _ in range(3):
        for g in graphs:
            g.replay()
        call(0, again, kept[0][3])
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
            a.fill_(0)
        torch.cuda.synchronize()
