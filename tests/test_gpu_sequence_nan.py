"""What is not finite in the 8-bit linear layer and in group normalisation: NaN before the activation, and of that what the activation makes, which is 0 for ReLU; the other rows' results as they were."""
import pytest

import test_gpu_group_norm as N
import test_gpu_linear_q8 as Q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("m", [1, 2, 20, 90])
def test_linear_q8(m, act):
    import torch
    import paper_1807_02037_amd as L
    k, n = 200, 72
    d = Q.make(torch, 2, m, k, n, True, True, "bf16", 0)
    ys = []
    for bad in (None, float("nan"), float("inf")):
        if bad is not None:
            d["x"][0, 7] = bad
            d["w"][5, 11] = -bad
        desc, wq, sw, ws, s = Q.setup(torch, L, d, m, k, n, act, 0)
        y = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        L.linear_q8_fwd(desc, *(d["x"].data_ptr(), wq.data_ptr(), sw.data_ptr(), d["bias"].data_ptr(), d["res"].data_ptr(), y.data_ptr(), ws.data_ptr()), s)
        torch.cuda.synchronize()
        ys.append(y)
    clean = [j for j in range(n) if j != 11]
    for y in ys[1:]:
        assert torch.equal(y[1:, clean], ys[0][1:, clean])
        for hit, res in ((y[0], d["res"][0]), (y[:, 11], d["res"][:, 11])):
            assert torch.equal(hit, res) if act == "relu" else hit.isnan().all()


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("n,s,c,groups", [(5, 1, 64, 4), (5, 1, 60, 4), (5, 40, 64, 4), (5, 40, 60, 4), (5, 3000, 64, 4)])
def test_group_norm(n, s, c, groups, act):
    import torch
    import paper_1807_02037_amd as L
    d = N.make(torch, 4, n, s, c, True, "bf16", 0)
    clean = N.call(torch, L, d, n, s, c, groups, act, 0)
    for bad in (float("nan"), float("-inf")):
        d["x"][2 * s, 20] = bad                                    # sample 2, group 1
        got = N.call(torch, L, d, n, s, c, groups, act, 0)
        torch.cuda.synchronize()
        for k in ("y", "dx"):
            a, b = got[k].reshape(n, s, groups, -1), clean[k].reshape(n, s, groups, -1).clone()
            hit = a[2, :, 1].clone()
            assert (hit == 0).all() if act == "relu" and k == "y" else hit.isnan().all()
            a[2, :, 1], b[2, :, 1] = 0, 0
            assert torch.equal(a, b), k
