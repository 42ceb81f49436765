"""Every tile, ring, split and join that the products of the language-model layers choose between, element by element: operands are small whole numbers, so that every
sum is exact in 32 bits in any order (a bound on the sums of magnitudes is checked), and every result has to be the exact one, rounded once.  Extents and reductions are no
multiples of the tiles; what lies between the rows, behind them and in the workspace is checked or poisoned."""
import pytest

from helpers import kernel_names
from test_gpu_dense_layers import dt, ptr, setup, space, stream

pytestmark = pytest.mark.gpu


def tile(bm, bn, ring, mode, dma=True, waves="2, 2"):
    return f"DenseTile<{bm}, {bn}, 64, {ring}, {waves}>, {mode}, {'true' if dma else 'false'}>"


def few(mode, rows, columns, kind="unsigned short"):
    return f"dense_few_kernel<{kind}, {mode}, {rows}, {columns}>"


def large(mode):
    return f"dense_large_kernel<{mode}>"


def f32(mode, edge, dma=True):
    return f"dense_f32_dma_kernel<{mode}, {edge}, {2 if edge == 128 else 5}>" if dma else f"dense_f32_kernel<{mode}, {edge}, false>"


def join(mode, kind="unsigned short"):
    return f"dense_join_kernel<{kind}, {mode}>"


FWD, GATED, DX, DW = range(4)
F = "float"
# m, k, n, elements between the rows; kernels that have to be among those launched: of the linear layer and the gated one in bf16, of both in fp32
SIZES = {
    "one_row_split": (1, 4104, 4104, 0, [few(FWD, 1, 128), join(FWD), tile(32, 128, 4, DX, waves="1, 4"), join(DX)], [few(GATED, 1, 128), join(GATED)],
                      [few(FWD, 1, 128, F), join(FWD, F)], [few(GATED, 1, 128, F), join(GATED, F)]),
    "two_rows_split": (2, 4104, 4104, 8, [few(FWD, 2, 128), join(FWD)], [few(GATED, 2, 128), join(GATED)], [few(FWD, 2, 128, F)], [few(GATED, 2, 128, F)]),
    "one_row_odd_split": (1, 3001, 5003, 3, [few(FWD, 1, 128), join(FWD)], [few(GATED, 1, 128), join(GATED)], [few(FWD, 1, 128, F)], [few(GATED, 1, 128, F)]),
    "one_row_32_columns": (1, 72, 8200, 0, [few(FWD, 1, 32)], [few(GATED, 1, 32)], [few(FWD, 1, 32, F)], [few(GATED, 1, 32, F)]),
    "one_row_64_columns": (1, 72, 16392, 8, [few(FWD, 1, 64)], [few(GATED, 1, 64)], [few(FWD, 1, 64, F)], [few(GATED, 1, 64, F)]),
    "two_rows_64_odd_columns": (2, 77, 16397, 3, [few(FWD, 2, 64)], [few(GATED, 2, 64)], [few(FWD, 2, 64, F)], [few(GATED, 2, 64, F)]),
    "four_rows": (4, 520, 4104, 0, [tile(64, 64, 5, FWD)], [tile(64, 128, 3, GATED)], [few(FWD, 4, 16, F)], [few(GATED, 4, 128, F), join(GATED, F)]),
    "eight_rows": (8, 520, 8201, 3, [tile(64, 128, 3, FWD, False)], [tile(64, 128, 3, GATED, False)], [few(FWD, 8, 128, F), join(FWD, F)], [f32(GATED, 128, False)]),
    "rows_of_32": (24, 2056, 8200, 0, [tile(32, 128, 4, FWD, waves="1, 4"), join(FWD)], [tile(64, 128, 3, GATED)], [f32(FWD, 64), join(FWD, F), f32(DX, 64)],
                   [f32(GATED, 128), join(GATED, F)]),
    "odd_split": (24, 2057, 1003, 3, [tile(64, 128, 3, FWD, False), join(FWD)], [tile(64, 128, 3, GATED, False), join(GATED)],
                  [f32(FWD, 64, False), f32(DX, 64, False), f32(DW, 128, False), join(FWD, F)], [f32(GATED, 128, False), join(GATED, F)]),
    "short_split": (100, 4000, 520, 8, [tile(64, 64, 5, FWD), join(FWD), tile(64, 64, 5, DX), tile(64, 128, 3, DW)], [tile(64, 128, 3, GATED), join(GATED)],
                    [f32(FWD, 64), f32(DX, 64), f32(DW, 128), join(FWD, F)], [f32(GATED, 128), join(GATED, F), join(DX, F)]),
    "tiles_64x128": (260, 520, 5200, 0, [tile(64, 128, 3, FWD), tile(64, 64, 5, DX), join(DX), tile(128, 128, 5, DW)],
                     [tile(128, 128, 5, GATED), tile(64, 128, 3, DX), join(DX)], [f32(FWD, 64), f32(DW, 64)], [f32(GATED, 128)]),
    "deep_128": (515, 4104, 4104, 8, [tile(128, 128, 5, FWD), tile(128, 128, 5, DX), tile(128, 128, 2, DW)], [tile(128, 128, 2, GATED)],
                 [f32(FWD, 128), f32(DX, 128), f32(DW, 128), join(FWD, F), join(DX, F)], [f32(GATED, 128), join(GATED, F)]),
    "tiles_128": (1030, 2056, 4104, 0, [tile(128, 128, 2, FWD), large(DW)], [tile(128, 128, 5, GATED), tile(128, 128, 2, DW)], [f32(DX, 128), f32(DW, 64)], [f32(GATED, 128)]),
    "odd_128": (2050, 1033, 4099, 3, [tile(128, 128, 2, FWD, False), tile(128, 128, 2, DX, False), tile(128, 128, 2, DW, False)], [tile(128, 128, 2, GATED, False)],
                [f32(FWD, 64, False), f32(DX, 128, False)], [f32(GATED, 128, False)]),
    "split_256": (2050, 4104, 4104, 8, [tile(128, 128, 5, FWD), large(DX)], [large(DX), join(DX), large(DW)], [f32(FWD, 128)], [f32(GATED, 128), f32(DX, 128), join(DX, F)]),
    "cut_256": (4091, 4104, 4088, 8, [large(FWD), tile(128, 128, 2, DX)], [large(GATED), large(DW)], [f32(FWD, 128), f32(DW, 128), join(DW, F)], [f32(GATED, 128)]),
    "long_reduction": (5000, 264, 264, 0, [tile(64, 128, 3, FWD), tile(64, 128, 3, DX), tile(64, 64, 5, DW), join(DW)], [tile(64, 64, 5, DW), join(DW)],
                       [f32(FWD, 64), f32(DW, 64), join(DW, F)], [f32(DW, 64), join(DW, F)]),
    "mixed": (1531, 1032, 2056, 0, [tile(128, 128, 5, FWD), tile(64, 128, 3, DX), tile(128, 128, 5, DW)], [tile(128, 128, 2, GATED), tile(128, 128, 5, DX), join(DX)],
              [f32(DW, 128), join(DW, F)], [f32(GATED, 128)]),
}
MARK = 12345.0


def whole_numbers(torch, seed, rows, cols, kind, pad, most):
    """Whole numbers from -most to most, rows cols + pad apart with NaN between them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.full((rows, cols + pad), float("nan"), device="cuda")
    t[:, :cols] = torch.randint(-most, most + 1, (rows, cols), generator=g, device="cuda").float()
    return t.to(kind)[:, :cols]


class Out:
    """An output with marks between its rows and in two rows behind them."""

    def __init__(self, torch, rows, cols, kind, pad):
        self.all = torch.full((rows + 2, cols + pad), MARK, dtype=kind, device="cuda")
        self.t = self.all[:rows, :cols]

    def data_ptr(self):
        return self.all.data_ptr()

    def check(self, want, what):
        got, ones = self.t, self.all.new_ones(())
        want = want.float().to(got.dtype)
        bad = (got != want).nonzero()
        assert not len(bad), (what, len(bad), bad[0].tolist(), got[tuple(bad[0])].item(), want[tuple(bad[0])].item())
        rest = self.all.clone()
        rest[:got.shape[0], :got.shape[1]] = MARK
        assert bool((rest == ones * MARK).all()), what + ": written beyond the rows"


def exact(a, b):
    """a @ b, whose terms' magnitudes stay below 2^24."""
    assert (a.abs() @ b.abs()).max().item() < 2 ** 24
    return a @ b


def reached(names, forms):
    for form in forms:
        assert any(form in v for v in names), (form, names)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_linear(size, dtype):
    torch, L, A = setup()
    m, k, n, pad, forms, _, forms32, _ = SIZES[size]
    kind, code = dt(torch, dtype), A.BF16 if dtype == "bf16" else A.F32
    x, w, res = (whole_numbers(torch, s, a, b, kind, pad, 2 - (s == 2)) for s, a, b in ((1, m, k), (2, k, n), (3, m, n)))
    dy = whole_numbers(torch, 4, m, n, kind, pad, 2)
    bias = whole_numbers(torch, 5, 1, n, torch.float32, 0, 9)
    d = L.linear_desc(m, n, k, act=A.ACT_RELU, dtype=code, wgrad_dtype=A.F32, ldx=k + pad, ldw=n + pad, ldy=n + pad, ldr=n + pad)
    plain = L.linear_desc(m, n, k, dtype=code, wgrad_dtype=code, ldx=k + pad, ldw=n + pad, ldy=n + pad)
    y, pre, dx, dx2 = (Out(torch, m, c, kind, pad) for c in (n, n, k, k))
    dw, dw2, db, db2 = Out(torch, k, n, torch.float32, pad), Out(torch, k, n, kind, pad), Out(torch, 1, n, torch.float32, 0), Out(torch, 1, n, torch.float32, 0)
    ws = space(torch, max(L.linear_workspace_bytes(e, v) for e in (d, plain) for v in (A.LINEAR_FWD, A.LINEAR_BWD)))

    def calls():
        s = stream(torch)
        L.linear_fwd(d, ptr(x), ptr(w), ptr(bias), ptr(res), ptr(y), ptr(pre), ptr(ws), s)
        L.linear_bwd(d, ptr(dy), ptr(x), ptr(w), ptr(pre), ptr(dx), ptr(dw), ptr(db), ptr(ws), s)
        L.linear_bwd(plain, ptr(dy), ptr(x), ptr(w), None, ptr(dx2), ptr(dw2), ptr(db2), ptr(ws), s)
    names = kernel_names(calls)
    X, W, R, D, B = (t.double() for t in (x, w, res, dy, bias))
    P = exact(X, W) + B
    pre.check(P, "pre")
    y.check(P.clamp(min=0) + R, "y")
    Z = D * (P > 0)
    dx.check(exact(Z, W.T), "dx")
    dw.check(exact(X.T, Z), "dw")
    db.check(Z.sum(0, keepdim=True), "db")
    dx2.check(exact(D, W.T), "dx without activation")
    dw2.check(exact(X.T, D), "dw without activation")
    db2.check(D.sum(0, keepdim=True), "db without activation")
    reached(names, forms if dtype == "bf16" else forms32)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_gated(size, dtype):
    torch, L, A = setup()
    m, k, f, pad, _, forms, _, forms32 = SIZES[size]
    kind, code = dt(torch, dtype), A.BF16 if dtype == "bf16" else A.F32
    x, wg, wu = (whole_numbers(torch, s, a, b, kind, pad, 2 - (s != 1)) for s, a, b in ((1, m, k), (2, k, f), (3, k, f)))
    dh = whole_numbers(torch, 4, m, f, kind, pad, 1)
    d = L.gated_desc(m, f, k, act=A.ACT_RELU, dtype=code, wgrad_dtype=A.F32, ldx=k + pad, ldw=f + pad, ldh=f + pad)
    h, g, u, dx, dx2 = (Out(torch, m, c, kind, pad) for c in (f, f, f, k, k))
    dws = [Out(torch, k, f, torch.float32, pad) for _ in range(4)]
    ws = space(torch, max(L.gated_workspace_bytes(d, v) for v in range(3)))

    def calls():
        s = stream(torch)
        L.gated_fwd(d, ptr(x), ptr(wg), ptr(wu), ptr(h), ptr(g), ptr(u), ptr(ws), s)
        L.gated_bwd(d, ptr(dh), ptr(x), ptr(wg), ptr(wu), ptr(g), ptr(u), ptr(dx), ptr(dws[0]), ptr(dws[1]), ptr(ws), s)
        L.gated_bwd(d, ptr(dh), ptr(x), ptr(wg), ptr(wu), None, None, ptr(dx2), ptr(dws[2]), ptr(dws[3]), ptr(ws), s)
    names = kernel_names(calls)
    X, WG, WU, D = (t.double() for t in (x, wg, wu, dh))
    G, U = exact(X, WG), exact(X, WU)
    assert (G * U).abs().max().item() < 2 ** 24
    h.check(G.clamp(min=0) * U, "h")
    g.check(G, "g")
    u.check(U, "u")
    for (gg, uu), dxs, (dwg, dwu), what in (((g.t.double(), u.t.double()), dx, dws[:2], "kept"), ((G, U), dx2, dws[2:], "computed again")):
        DG, DU = ((D * v).float().to(kind).double() for v in (uu * (gg > 0), gg.clamp(min=0)))     # rounded to the storage type where they enter the products
        assert (DG.abs() @ WG.abs().T + DU.abs() @ WU.abs().T).max().item() < 2 ** 24
        dxs.check(DG @ WG.T + DU @ WU.T, "dx, " + what)
        dwg.check(exact(X.T, DG), "dwg, " + what)
        dwu.check(exact(X.T, DU), "dwu, " + what)
    reached(names, forms if dtype == "bf16" else forms32)
