"""The 8-bit linear layer where the scales' product, or a sum's with one of them, leaves the range of 32 bits and the result need not: every kernel, split sums too."""
import numpy as np
import pytest

import test_gpu_linear_q8 as Q
from layer_oracle import U, f64

pytestmark = pytest.mark.gpu

# m, k, n: one and two rows, blocks of 16 and 32 columns, tiles in one piece, tiles in splits, one large
SHAPES = [(1, 64, 40), (2, 512, 40), (5, 300, 50), (40, 1000, 70), (20, 256, 4200), (70, 300, 24), (100, 8192, 40), (300, 400, 300), (2100, 64, 2050)]
# powers of ten of rows and of columns, by turns
ROWS, COLUMNS = [38, -30, 0, -36, 20, 30, -38], [5, -14, 37, -36, -20, 0, -8]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_scales_at_their_ends(m, k, n, dtype):
    import torch
    import paper_1807_02037_amd as L
    d = Q.make(torch, 1, m, k, n, False, False, dtype, 0)
    x, w = d["x"].double().cpu(), d["w"].double().cpu()
    x, w = x / x.abs().amax(1, keepdim=True), w / w.abs().amax(0, keepdim=True)
    x[::3] = torch.where(torch.arange(k) % 2 == 0, 1.0, -1.0).double()
    w[:, ::3] = 1.0                                                # sums of 0 with the rows of signs by turns
    x *= 10.0 ** torch.tensor([ROWS[i % 7] for i in range(m)], dtype=torch.float64)[:, None]
    w *= 10.0 ** torch.tensor([COLUMNS[j % 7] for j in range(n)], dtype=torch.float64)
    d["x"], d["w"] = x.to(d["kind"]).cuda(), w.to(d["kind"]).cuda()
    desc, wq, sw, ws, s = Q.setup(torch, L, d, m, k, n, "none", 0)
    y = torch.full((m, n), 777.0, dtype=d["kind"], device="cuda")
    L.linear_q8_fwd(desc, d["x"].data_ptr(), wq.data_ptr(), sw.data_ptr(), None, None, y.data_ptr(), ws.data_ptr(), s)
    torch.cuda.synchronize()
    xq, _ = Q.steps(f64(d["x"]))
    wsteps, _ = Q.steps(f64(d["w"]).T)
    # the scales as they are given, in 32 bits
    scales = (np.abs(f64(d["x"])).max(1) / 127).astype(np.float32).astype(float), f64(sw)
    sums = xq @ wsteps.T
    want = sums * scales[0][:, None] * scales[1]
    assert (sums[0, ::3] == 0).all()
    # the scale of a row is within 2 units of the quotient, or 2^-149; the sum, the scales' product and the result are rounded, a small one to a multiple of 2^-149 and to its type once more
    e = 6 * Q.U32 * np.abs(want) + np.abs(sums) * scales[1] * 2.0 ** -149 + 2.0 ** -149
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    allowed = e + U[d["kind"]] * np.abs(want) + tiny
    top = float(torch.finfo(d["kind"]).max)
    got = f64(y)
    over = np.abs(want) + allowed >= top                           # may be infinite, and has to be beyond
    assert not np.isnan(got).any()
    assert (np.abs(got - want)[~over] <= allowed[~over]).all(), np.argwhere(~over & ~(np.abs(got - want) <= allowed))[0]
    assert (np.sign(got[over]) == np.sign(want[over])).all() and (np.abs(got[over]) >= np.minimum(np.abs(want[over]) - allowed[over], top)).all()
    assert (got[sums == 0] == 0).all()
