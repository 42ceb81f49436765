"""Values and slopes of the activations at finite arguments as large as the types hold: the limits, and no NaN from a product of nothing with what overflows."""
import pytest

import layer_oracle as O
from test_gpu_dense_layers import dt, out, ptr, setup, space, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", range(5))
def test_finite_arguments(act, dtype):
    torch, L, A = setup()
    kind, code = dt(torch, dtype), A.BF16 if dtype == "bf16" else A.F32
    most = torch.finfo(kind).max
    v = [s * a for a in (0.0, 100.0, 1e4, 1e7, 1e13, 1.8e19, 2e19, 1e25, 1e38, most) for s in (1, -1)]
    n = len(v)
    w, x, dy = torch.tensor([v], device="cuda").to(kind), torch.ones(1, 1, device="cuda").to(kind), torch.ones(1, n, device="cuda").to(kind)
    pre, y, h, db = out(torch, 1, n, kind), out(torch, 1, n, kind), out(torch, 1, n, kind), out(torch, 1, n, torch.float32)
    d = L.linear_desc(1, n, 1, act=act, dtype=code)
    ws = space(torch, max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD)))
    L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(y), ptr(pre), ptr(ws), stream(torch))
    L.linear_bwd(d, ptr(dy), ptr(x), ptr(w), ptr(pre), None, None, ptr(db), ptr(ws), stream(torch))
    torch.cuda.synchronize()
    assert torch.equal(pre, w)
    name = O.ACTS[act]
    for j, a in enumerate(O.f64(w)[0].tolist()):
        # beyond 100 every activation is its argument or nothing, and its slope 1 or 0, to more digits than 32 bits hold
        value, slope = (a, 1.0) if a > 0 or name == "none" else (0.0, 0.0)
        if a == 0:
            slope = {"none": 1.0, "relu": 0.0}.get(name, 0.5)
        assert y[0, j].item() == value and abs(db[0, j].item() - slope) <= 2.0 ** -22, (name, a, y[0, j].item(), db[0, j].item())
    # the gated projection's gradients use the same value and slope: dwg = dg and dwu = du with one row and x = 1
    g = L.gated_desc(1, n, 1, act=act, dtype=code)
    gws = space(torch, max(L.gated_workspace_bytes(g, c) for c in range(3)))
    one, dwg, dwu = torch.ones(1, n, device="cuda").to(kind), out(torch, 1, n, torch.float32), out(torch, 1, n, torch.float32)
    L.gated_fwd(g, ptr(x), ptr(w), ptr(one), ptr(h), None, None, ptr(gws), stream(torch))
    assert torch.equal(h, y)
    for kept in ((ptr(w), ptr(one)), (None, None)):
        L.gated_bwd(g, ptr(dy), ptr(x), ptr(w), ptr(one), *kept, None, ptr(dwg), ptr(dwu), ptr(gws), stream(torch))
        torch.cuda.synchronize()
        assert torch.equal(dwu, y.float()) and bool((dwg - db).abs().max() <= 2.0 ** -8)
