"""Linear layer and gated projection on the GPU against fp64: sizes from one element on, ragged and odd ones, row pitches with NaN between the
rows, every activation, optional operands, both types."""
import numpy as np
import pytest

import layer_oracle as O
from helpers import kernel_names

pytestmark = pytest.mark.gpu

# m, k, n: single elements, tokens one by one, tiles not filled, filled and passed by one, lengths that no vector divides
SIZES = [(1, 1, 1), (1, 64, 64), (2, 7, 9), (1, 520, 136), (3, 8, 8), (8, 264, 1032), (17, 96, 260), (33, 65, 129), (64, 1000, 77), (127, 64, 128),
         (129, 200, 136), (256, 136, 264), (300, 264, 328), (515, 72, 520),
         (260, 393, 94), (9, 131, 135), (140, 7, 300), (7, 200, 5), (131, 193, 193)]
DTYPES = ["bf16", "fp32"]


def setup():
    import torch
    import paper_1807_02037_amd as L
    return torch, L, L.abi


def dt(torch, name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def matrix(torch, seed, rows, cols, dtype, pad=0, scale=1.0):
    """Rows cols + pad apart, with NaN between them."""
    g = torch.Generator().manual_seed(seed)
    t = torch.full((rows, cols + pad), float("nan"), dtype=torch.float32)
    t[:, :cols] = torch.randn(rows, cols, generator=g) * scale
    return t.to(dtype).cuda()[:, :cols]


def out(torch, rows, cols, dtype, pad=0):
    """An output whose elements, and those between its rows, hold a number that no result is."""
    return torch.full((rows, cols + pad), 12345.0, dtype=dtype, device="cuda")[:, :cols]


def whole(t):
    return t.as_strided((t.shape[0], t.stride(0)), t.stride()) if t.shape[0] > 1 else t


def untouched(t):
    """Nothing was written between the rows."""
    pad = whole(t)[:, t.shape[1]:].float()
    return bool((pad == pad.new_tensor(12345.0).to(t.dtype).float()).all())


def ptr(t):
    return None if t is None else t.data_ptr()


def space(torch, nbytes):
    return torch.full((max(nbytes, 16),), 255, dtype=torch.uint8, device="cuda")      # NaN in every type


def near(got, want, bound, what):
    off = np.abs(O.f64(got) - want)
    bad = ~(off <= bound + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0], off[bad][0], np.broadcast_to(bound, off.shape)[bad][0])


def stream(torch):
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_linear(i, dtype):
    torch, L, A = setup()
    m, k, n = SIZES[i]
    kind = dt(torch, dtype)
    code = A.BF16 if dtype == "bf16" else A.F32
    name = O.ACTS[i % 5]
    pad = (0, 8, 3)[i % 3]
    x, w = matrix(torch, i, m, k, kind, pad), matrix(torch, i + 100, k, n, kind, (0, 16, 5)[i % 3], k ** -0.5)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(i)).cuda() if i % 4 else None
    res = matrix(torch, i + 200, m, n, kind, (8, 0, 1)[i % 3]) if i % 2 else None
    y, pre = out(torch, m, n, kind, pad), out(torch, m, n, kind, pad)
    d = L.linear_desc(m, n, k, act=i % 5, dtype=code, ldx=k + pad, ldw=n + (0, 16, 5)[i % 3], ldy=n + pad, ldr=n + (8, 0, 1)[i % 3])
    ws = space(torch, L.linear_workspace_bytes(d, A.LINEAR_FWD))
    L.linear_fwd(d, ptr(x), ptr(w), ptr(bias), ptr(res), ptr(y), ptr(pre), ptr(ws), stream(torch))
    torch.cuda.synchronize()
    want_y, want_pre, e_y, e_pre = O.linear_fwd(name, O.f64(x), O.f64(w), None if bias is None else O.f64(bias), None if res is None else O.f64(res), kind)
    near(pre, want_pre, e_pre, "pre")
    near(y, want_y, e_y, "y")
    assert untouched(y) and untouched(pre)
    # the same without pre gives the same bits
    again = out(torch, m, n, kind, pad)
    L.linear_fwd(d, ptr(x), ptr(w), ptr(bias), ptr(res), ptr(again), None, ptr(ws), stream(torch))
    assert torch.equal(again, y)

    dy = matrix(torch, i + 300, m, n, kind, pad)
    for wcode, wkind in ((A.F32, torch.float32),) + (((A.BF16, torch.bfloat16),) if dtype == "bf16" else ()):
        d = L.linear_desc(m, n, k, act=i % 5, dtype=code, wgrad_dtype=wcode, ldx=k + pad, ldw=n + (0, 16, 5)[i % 3], ldy=n + pad)
        dx, dw, db = out(torch, m, k, kind, pad), out(torch, k, n, wkind, (0, 16, 5)[i % 3]), out(torch, 1, n, torch.float32)
        ws = space(torch, L.linear_workspace_bytes(d, A.LINEAR_BWD))
        args = (ptr(dy), ptr(x), ptr(w), ptr(pre) if i % 5 else None)
        L.linear_bwd(d, *args, ptr(dx), ptr(dw), ptr(db), ptr(ws), stream(torch))
        torch.cuda.synchronize()
        want = O.linear_bwd(name, O.f64(dy), O.f64(x), O.f64(w), O.f64(pre), kind, wkind)
        near(dx, want[0], want[1], "dx")
        near(dw, want[2], want[3], "dw")
        near(db[0], want[4], want[5], "db")
        assert untouched(dx) and untouched(dw)
        # each output alone has the same bits
        for keep in range(3):
            one = [out(torch, m, k, kind, pad), out(torch, k, n, wkind, (0, 16, 5)[i % 3]), out(torch, 1, n, torch.float32)]
            L.linear_bwd(d, *args, *[ptr(t) if j == keep else None for j, t in enumerate(one)], ptr(ws), stream(torch))
            assert torch.equal(one[keep], (dx, dw, db)[keep])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_gated(i, dtype):
    torch, L, A = setup()
    m, k, f = SIZES[i]
    kind = dt(torch, dtype)
    code = A.BF16 if dtype == "bf16" else A.F32
    name, pad = O.ACTS[(i + 2) % 5], (3, 0, 8)[i % 3]
    x = matrix(torch, i, m, k, kind, pad)
    both = matrix(torch, i + 100, k, 2 * f, kind, 0, k ** -0.5)     # wg and wu are halves of one matrix
    wg, wu = both[:, :f], both[:, f:]
    g, u, h = (out(torch, m, f, kind, pad) for _ in range(3))
    d = L.gated_desc(m, f, k, act=(i + 2) % 5, dtype=code, ldx=k + pad, ldw=2 * f, ldh=f + pad)
    ws = space(torch, L.gated_workspace_bytes(d, A.GATED_FWD))
    L.gated_fwd(d, ptr(x), ptr(wg), ptr(wu), ptr(h), ptr(g), ptr(u), ptr(ws), stream(torch))
    torch.cuda.synchronize()
    want = O.gated_fwd(name, O.f64(x), O.f64(wg), O.f64(wu), kind)
    near(h, want[0], want[3], "h")
    near(g, want[1], want[4], "g")
    near(u, want[2], want[5], "u")
    assert untouched(h) and untouched(g) and untouched(u)
    again = out(torch, m, f, kind, pad)
    L.gated_fwd(d, ptr(x), ptr(wg), ptr(wu), ptr(again), None, None, ptr(ws), stream(torch))
    assert torch.equal(again, h)

    dh = matrix(torch, i + 200, m, f, kind, pad)
    for wcode, wkind in ((A.F32, torch.float32),) + (((A.BF16, torch.bfloat16),) if dtype == "bf16" else ()):
        d = L.gated_desc(m, f, k, act=(i + 2) % 5, dtype=code, wgrad_dtype=wcode, ldx=k + pad, ldw=2 * f, ldh=f + pad)
        for kept in (True, False):
            dx, dboth = out(torch, m, k, kind, pad), out(torch, k, 2 * f, wkind)
            ws = space(torch, L.gated_workspace_bytes(d, A.GATED_BWD if kept else A.GATED_BWD_RECOMPUTE))
            args = (ptr(dh), ptr(x), ptr(wg), ptr(wu)) + ((ptr(g), ptr(u)) if kept else (None, None))
            L.gated_bwd(d, *args, ptr(dx), ptr(dboth), ptr(dboth[:, f:]), ptr(ws), stream(torch))
            torch.cuda.synchronize()
            e_dx = O.gated_bwd(name, O.f64(dh), O.f64(x), O.f64(wg), O.f64(wu), O.f64(g) if kept else None, O.f64(u) if kept else None, kind, wkind)
            near(dx, e_dx[0], e_dx[1], "dx")
            near(dboth[:, :f], *e_dx[2][0], "dwg")
            near(dboth[:, f:], *e_dx[2][1], "dwu")
            assert untouched(dx)
            one = out(torch, m, k, kind, pad)
            L.gated_bwd(d, *args, ptr(one), None, None, ptr(ws), stream(torch))
            assert torch.equal(one, dx)
            two = out(torch, k, 2 * f, wkind)
            L.gated_bwd(d, *args, None, ptr(two), ptr(two[:, f:]), ptr(ws), stream(torch))
            assert torch.equal(two, dboth)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(dtype):
    """Weight and bias gradients of no rows are zeros; nothing else is written."""
    torch, L, A = setup()
    kind, code = dt(torch, dtype), A.BF16 if dtype == "bf16" else A.F32
    k, n = 24, 40
    d = L.linear_desc(0, n, k, act=A.ACT_SILU, dtype=code, wgrad_dtype=code, ldw=n + 8)
    w, dw, db, y = matrix(torch, 1, k, n, kind, 8), out(torch, k, n, kind, 8), out(torch, 1, n, torch.float32), out(torch, 1, n, kind)
    L.linear_fwd(d, ptr(y), ptr(w), None, None, ptr(y), None, None, stream(torch))
    L.linear_bwd(d, ptr(y), ptr(y), ptr(w), ptr(y), ptr(y), ptr(dw), ptr(db), None, stream(torch))
    g = L.gated_desc(0, n, k, dtype=code, wgrad_dtype=A.F32, ldw=n + 8)
    dwg, dwu = out(torch, k, n, torch.float32, 8), out(torch, k, n, torch.float32, 8)
    L.gated_fwd(g, ptr(y), ptr(w), ptr(w), ptr(y), None, None, None, stream(torch))
    L.gated_bwd(g, ptr(y), ptr(y), ptr(w), ptr(w), None, None, ptr(y), ptr(dwg), ptr(dwu), None, stream(torch))
    torch.cuda.synchronize()
    for t in (dw, db, dwg, dwu):
        assert not t.any() and untouched(t)
    assert bool((y == y.new_tensor(12345.0)).all())


def test_residual_in_place_and_another_stream():
    torch, L, A = setup()
    m, k, n = 200, 136, 264
    x, w, res = matrix(torch, 1, m, k, torch.bfloat16), matrix(torch, 2, k, n, torch.bfloat16, 0, k ** -0.5), matrix(torch, 3, m, n, torch.bfloat16)
    d = L.linear_desc(m, n, k, act=A.ACT_GELU)
    y = out(torch, m, n, torch.bfloat16)
    L.linear_fwd(d, ptr(x), ptr(w), None, ptr(res), ptr(y), None, None, stream(torch))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    late = res.clone()
    torch.cuda.synchronize()
    L.linear_fwd(d, ptr(x), ptr(w), None, ptr(late), ptr(late), None, None, s.cuda_stream)
    s.synchronize()
    assert torch.equal(late, y)


def test_infinities_stay_in_their_rows():
    """An infinite or NaN input reaches its own row of y and dx, and no other; beside it everything is finite."""
    torch, L, A = setup()
    m, k, n = 70, 72, 136
    x, w = matrix(torch, 1, m, k, torch.bfloat16), matrix(torch, 2, k, n, torch.bfloat16)
    x[5, 7], x[69, 71] = float("inf"), float("nan")
    y = out(torch, m, n, torch.bfloat16)
    L.linear_fwd(L.linear_desc(m, n, k), ptr(x), ptr(w), None, None, ptr(y), None, None, stream(torch))
    fine = torch.isfinite(y.float()).all(1)
    assert not torch.isfinite(y[5].float()).any() and torch.isnan(y[69]).all()
    assert fine.sum() == m - 2


def test_gradient_is_the_slope_of_the_loss():
    """fp32: the loss sum(y c) moves by the gradient times a small step, by central differences in the direction of the gradient."""
    torch, L, A = setup()
    m, k, n = 9, 20, 12
    x, w, c = (matrix(torch, s, a, b, torch.float32) for s, a, b in ((1, m, k), (2, k, n), (3, m, n)))
    for code in range(5):
        d = L.linear_desc(m, n, k, act=code, dtype=A.F32)
        ws = space(torch, L.linear_workspace_bytes(d, A.LINEAR_BWD))
        y, pre = out(torch, m, n, torch.float32), out(torch, m, n, torch.float32)

        def loss(xx, ww):
            L.linear_fwd(d, ptr(xx), ptr(ww), None, None, ptr(y), ptr(pre), ptr(ws), stream(torch))
            return (y.double() * c.double()).sum().item()
        loss(x, w)
        dx, dw = out(torch, m, k, torch.float32), out(torch, k, n, torch.float32)
        L.linear_bwd(d, ptr(c), ptr(x), ptr(w), ptr(pre), ptr(dx), ptr(dw), None, ptr(ws), stream(torch))
        for grad, shift in ((dx, lambda s: (x + s * dx, w)), (dw, lambda s: (x, w + s * dw))):
            step = 2.0 ** -9 / grad.norm().item()
            slope = (loss(*shift(step)) - loss(*shift(-step))) / (2 * step)
            want = grad.double().square().sum().item()
            # third derivatives times step^2, and fp32 sums of the loss over 2 step; kinks of ReLU are crossed by few elements
            assert abs(slope - want) <= (2e-2 if code == A.ACT_RELU else 5e-3) * want, (code, slope, want)


def test_same_bits_again():
    torch, L, A = setup()
    m, k, f = 700, 264, 520
    x, wg, wu, dh = (matrix(torch, s, a, b, torch.bfloat16) for s, a, b in ((1, m, k), (2, k, f), (3, k, f), (4, m, f)))
    d = L.gated_desc(m, f, k, wgrad_dtype=A.F32)
    ws = space(torch, L.gated_workspace_bytes(d, A.GATED_BWD_RECOMPUTE))
    seen = []
    for _ in range(3):
        dx, dwg, dwu = out(torch, m, k, torch.bfloat16), out(torch, k, f, torch.float32), out(torch, k, f, torch.float32)
        L.gated_bwd(d, ptr(dh), ptr(x), ptr(wg), ptr(wu), None, None, ptr(dx), ptr(dwg), ptr(dwu), ptr(ws), stream(torch))
        seen.append((dx, dwg, dwu))
    torch.cuda.synchronize()
    for later in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], later))


def test_rows_beyond_32_bit_offsets():
    """Rows so far apart that the last ones lie beyond 2^32 bytes and 2^31 elements."""
    torch, L, A = setup()
    m, k, n, pitch = 2200, 64, 128, 1 << 20
    big = torch.empty(m * pitch, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((m, k), (pitch, 1))
    x.copy_(matrix(torch, 1, m, k, torch.bfloat16))
    w = matrix(torch, 2, k, n, torch.bfloat16, 0, 0.125)
    y = big.as_strided((m, n), (pitch, 1), 1024)
    d = L.linear_desc(m, n, k, ldx=pitch, ldy=pitch)
    L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(y), None, None, stream(torch))
    want, _, e, _ = O.linear_fwd("none", O.f64(x), O.f64(w), None, None, torch.bfloat16)
    near(y, want, e, "y")
    dw, dx = out(torch, k, n, torch.float32), big.as_strided((m, k), (pitch, 1), 4096)
    ws = space(torch, L.linear_workspace_bytes(d, A.LINEAR_BWD))
    L.linear_bwd(d, ptr(y), ptr(x), ptr(w), None, ptr(dx), ptr(dw), None, ptr(ws), stream(torch))
    wdx, e_dx, wdw, e_dw, _, _ = O.linear_bwd("none", O.f64(y), O.f64(x), O.f64(w), None, torch.bfloat16, torch.float32)
    near(dx, wdx, e_dx, "dx")
    near(dw, wdw, e_dw, "dw")


def test_wide_pitches_in_fp32():
    """Rows of 2^21 elements and more, whose tiles have no 32-bit offsets."""
    torch, L, A = setup()
    m, k, n, pitch = 150, 40, 72, (1 << 21) + 3
    big = torch.empty(m * pitch, device="cuda")
    x, y, dx = (big.as_strided((m, c), (pitch, 1), at) for c, at in ((k, 0), (n, 1000), (k, 5000)))
    x.copy_(matrix(torch, 1, m, k, torch.float32))
    w = matrix(torch, 2, k, n, torch.float32)
    d = L.linear_desc(m, n, k, dtype=A.F32, ldx=pitch, ldy=pitch)
    ws = space(torch, max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD)))
    L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(y), None, ptr(ws), stream(torch))
    want, _, e, _ = O.linear_fwd("none", O.f64(x), O.f64(w), None, None, torch.float32)
    near(y, want, e, "y")
    dw = out(torch, k, n, torch.float32)
    L.linear_bwd(d, ptr(y), ptr(x), ptr(w), None, ptr(dx), ptr(dw), None, ptr(ws), stream(torch))
    wdx, e_dx, wdw, e_dw, _, _ = O.linear_bwd("none", O.f64(y), O.f64(x), O.f64(w), None, torch.float32, torch.float32)
    near(dx, wdx, e_dx, "dx")
    near(dw, wdw, e_dw, "dw")


def test_wide_pitches_in_bf16():
    """The same in bf16, through registers: pitches of 2^21 elements and more."""
    torch, L, A = setup()
    m, k, n, pitch = 300, 72, 136, (1 << 21) + 8
    big = torch.empty(m * pitch, dtype=torch.bfloat16, device="cuda")
    x, y, dx = (big.as_strided((m, c), (pitch, 1), at) for c, at in ((k, 0), (n, 1024), (k, 4096)))
    x.copy_(matrix(torch, 1, m, k, torch.bfloat16))
    w = matrix(torch, 2, k, n, torch.bfloat16, 0, 0.125)
    d = L.linear_desc(m, n, k, ldx=pitch, ldy=pitch)
    ws = space(torch, max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD)))
    L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(y), None, ptr(ws), stream(torch))
    want, _, e, _ = O.linear_fwd("none", O.f64(x), O.f64(w), None, None, torch.bfloat16)
    near(y, want, e, "y")
    dw, db = out(torch, k, n, torch.float32), out(torch, 1, n, torch.float32)
    L.linear_bwd(d, ptr(y), ptr(x), ptr(w), None, ptr(dx), ptr(dw), ptr(db), ptr(ws), stream(torch))
    wdx, e_dx, wdw, e_dw, wdb, e_db = O.linear_bwd("none", O.f64(y), O.f64(x), O.f64(w), None, torch.bfloat16, torch.float32)
    near(dx, wdx, e_dx, "dx")
    near(dw, wdw, e_dw, "dw")
    near(db[0], wdb, e_db, "db")


def test_bias_gradient_of_many_rows():
    """More rows than chunks of the smallest size; the sums of a column of ones are exact."""
    torch, L, A = setup()
    m, k, n = 70001, 8, 24
    dy = torch.ones(m, n, dtype=torch.bfloat16, device="cuda")
    dy[:, 3] = -2.0
    x, db = torch.ones(m, k, dtype=torch.bfloat16, device="cuda"), out(torch, 1, n, torch.float32)
    dw = out(torch, k, n, torch.float32)
    d = L.linear_desc(m, n, k)
    ws = space(torch, L.linear_workspace_bytes(d, A.LINEAR_BWD))
    L.linear_bwd(d, ptr(dy), ptr(x), None, None, None, ptr(dw), ptr(db), ptr(ws), stream(torch))
    want = torch.full((n,), float(m), device="cuda")
    want[3] = -2.0 * m
    assert torch.equal(db[0], want) and torch.equal(dw, want.expand(k, n))


@pytest.mark.parametrize("act", range(5))
def test_whole_large_tiles(act):
    """Several 256 x 256 tiles, whole and cut, of every product, against fp64 in norm: each element is rounded once, and what enters the backward products once more."""
    torch, L, A = setup()
    m, k, n = 4091, 4096, 4096
    x, w, res = matrix(torch, 1, m, k, torch.bfloat16), matrix(torch, 2, k, n, torch.bfloat16, 0, k ** -0.5), matrix(torch, 3, m, n, torch.bfloat16)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(4)).cuda()
    d = L.linear_desc(m, n, k, act=act)
    ws = space(torch, max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD)))
    y, pre, dx, dw, db = (out(torch, *s, t) for s, t in (((m, n), torch.bfloat16), ((m, n), torch.bfloat16), ((m, k), torch.bfloat16), ((k, n), torch.float32),
                                                         ((1, n), torch.float32)))
    L.linear_fwd(d, ptr(x), ptr(w), ptr(bias), ptr(res), ptr(y), ptr(pre), ptr(ws), stream(torch))
    names = kernel_names(lambda: L.linear_bwd(d, ptr(res), ptr(x), ptr(w), ptr(pre), ptr(dx), ptr(dw), ptr(db), ptr(ws), stream(torch)))
    assert sum("dense_large_kernel" in v for v in names) == 2, names
    X, W, R, B = x.double(), w.double(), res.double(), bias.double()
    P = X @ W + B
    name = O.ACTS[act]

    def same(got, want, u, what):
        assert ((got.double() - want).norm() / want.norm()).item() <= u, what
    Y, _ = O.act(name, P.cpu().numpy())
    same(pre, P, 2.0 ** -8, "pre")
    same(y, torch.from_numpy(Y).cuda() + R, 2.0 ** -8, "y")
    D = R * torch.from_numpy(O.act(name, O.f64(pre))[1]).cuda()
    same(dx, D @ W.T, 2.0 ** -7, "dx")
    same(dw, X.T @ D, 2.0 ** -8 if act else 1e-5, "dw")
    same(db[0], D.sum(0), 1e-5, "db")
    g = L.gated_desc(m, n, k, act=act)
    gws = space(torch, max(L.gated_workspace_bytes(g, c) for c in range(3)))
    w2 = matrix(torch, 5, k, n, torch.bfloat16, 0, k ** -0.5)
    h, dwg, dwu = out(torch, m, n, torch.bfloat16), out(torch, k, n, torch.float32), out(torch, k, n, torch.float32)
    L.gated_fwd(g, ptr(x), ptr(w), ptr(w2), ptr(h), None, None, ptr(gws), stream(torch))
    L.gated_bwd(g, ptr(res), ptr(x), ptr(w), ptr(w2), None, None, ptr(dx), ptr(dwg), ptr(dwu), ptr(gws), stream(torch))
    W2 = w2.double()
    G, U = X @ W, X @ W2
    a, s = (torch.from_numpy(v).cuda() for v in O.act(name, G.cpu().numpy()))
    DG, DU = R * U * s, R * a
    same(h, a * U, 2.0 ** -8, "h")
    same(dx, DG @ W.T + DU @ W2.T, 2.0 ** -7, "gated dx")
    same(dwg, X.T @ DG, 2.0 ** -8, "dwg")
    same(dwu, X.T @ DU, 2.0 ** -8, "dwu")


def test_replays_of_a_captured_step():
    """Forward and backward captured into a graph, replayed between eager work: each replay has the eager bits for its inputs."""
    torch, L, A = setup()
    m, k, n = 96, 200, 312
    x, w = matrix(torch, 1, m, k, torch.bfloat16), matrix(torch, 2, k, n, torch.bfloat16, 0, k ** -0.5)
    bias = torch.randn(n, device="cuda")
    d = L.linear_desc(m, n, k, act=A.ACT_SILU)
    need = max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD))

    def buffers():
        return [out(torch, m, n, torch.bfloat16), out(torch, m, n, torch.bfloat16), out(torch, m, k, torch.bfloat16), out(torch, k, n, torch.float32),
                out(torch, 1, n, torch.float32), space(torch, need)]

    def step(b):
        s = stream(torch)
        L.linear_fwd(d, ptr(x), ptr(w), ptr(bias), None, ptr(b[0]), ptr(b[1]), ptr(b[5]), s)
        L.linear_bwd(d, ptr(b[0]), ptr(x), ptr(w), ptr(b[1]), ptr(b[2]), ptr(b[3]), ptr(b[4]), ptr(b[5]), s)
    eager, taped = buffers(), buffers()
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(taped)
    for i in range(4):
        x.copy_(matrix(torch, 10 + i, m, k, torch.bfloat16))
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager[:5], taped[:5])), i
