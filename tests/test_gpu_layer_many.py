"""Calls of more work-groups than one grid holds (2^32 threads): rows, columns and classes by the hundred million, narrow enough to fit."""
import pytest

from test_gpu_dense_layers import ptr, setup, space, stream

pytestmark = pytest.mark.gpu


def same(torch, got, want, what):
    """Equal, a piece at a time; want(from, to) makes a piece."""
    for i in range(0, got.shape[0], 1 << 27):
        j = min(i + (1 << 27), got.shape[0])
        bad = (got[i:j] != want(i, j)).nonzero()
        assert not len(bad), (what, i + bad[0].item(), len(bad))


def test_linear_of_many_rows():
    """2^30 rows and more of one input and one output: 2^24 tiles of 64 rows."""
    torch, L, A = setup()
    for kind, code in ((torch.bfloat16, A.BF16), (torch.float32, A.F32)):
        m = (1 << 30) + 70
        x = torch.empty(m, dtype=kind, device="cuda")
        for i in range(0, m, 1 << 27):
            x[i:i + (1 << 27)] = (torch.arange(i, min(i + (1 << 27), m), device="cuda") % 31 - 15).to(kind)
        w = torch.full((1,), 3.0, device="cuda").to(kind)
        y, dx = torch.full((m,), 99.0, dtype=kind, device="cuda"), torch.full((m,), 99.0, dtype=kind, device="cuda")
        d = L.linear_desc(m, 1, 1, dtype=code)
        ws = space(torch, max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD)))
        L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(y), None, ptr(ws), stream(torch))
        L.linear_bwd(d, ptr(x), ptr(x), ptr(w), None, ptr(dx), None, None, ptr(ws), stream(torch))
        torch.cuda.synchronize()
        same(torch, y, lambda i, j: x[i:j] * 3, "y")
        same(torch, dx, lambda i, j: x[i:j] * 3, "dx")


def test_linear_of_many_columns():
    """One row of 2^29 outputs and more: 2^23 work-groups of 512 threads; the bias gradient sums 2^24 groups of columns, the weight gradient is as long."""
    torch, L, A = setup()
    n = (1 << 29) + 40
    for kind, code in ((torch.bfloat16, A.BF16), (torch.float32, A.F32)):
        w = torch.empty(n, dtype=kind, device="cuda")
        for i in range(0, n, 1 << 27):
            w[i:i + (1 << 27)] = (torch.arange(i, min(i + (1 << 27), n), device="cuda") % 29 - 14).to(kind)
        x, y = torch.full((1,), 5.0, device="cuda").to(kind), torch.full((n,), 99.0, dtype=kind, device="cuda")
        d = L.linear_desc(1, n, 1, dtype=code)
        ws = space(torch, max(L.linear_workspace_bytes(d, A.LINEAR_FWD), L.linear_workspace_bytes(d, A.LINEAR_BWD)))
        L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(y), None, ptr(ws), stream(torch))
        dw, db = torch.full((n,), 99.0, device="cuda"), torch.full((n,), 99.0, device="cuda")
        L.linear_bwd(d, ptr(w), ptr(x), ptr(w), None, None, ptr(dw), ptr(db), ptr(ws), stream(torch))
        torch.cuda.synchronize()
        same(torch, y, lambda i, j: w[i:j] * 5, "y")
        same(torch, dw, lambda i, j: w[i:j].float() * 5, "dw")
        same(torch, db, lambda i, j: w[i:j].float(), "db")


def test_weight_gradient_of_many_inputs():
    """2^30 inputs, one output, one row: 2^24 tiles of 64 rows of dw."""
    torch, L, A = setup()
    k = 1 << 30
    x = torch.empty(k, dtype=torch.bfloat16, device="cuda")
    for i in range(0, k, 1 << 27):
        x[i:i + (1 << 27)] = (torch.arange(i, i + (1 << 27), device="cuda") % 31 - 15).to(torch.bfloat16)
    dy, dw = torch.full((1,), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((k,), 99.0, device="cuda")
    d = L.linear_desc(1, 1, k)
    ws = space(torch, L.linear_workspace_bytes(d, A.LINEAR_BWD))
    L.linear_bwd(d, ptr(dy), ptr(x), None, None, None, ptr(dw), None, ptr(ws), stream(torch))
    torch.cuda.synchronize()
    same(torch, dw, lambda i, j: x[i:j].float() * 7, "dw")


def test_zeros_of_many_elements():
    """Weight gradients of no rows with more than 2^32 elements."""
    torch, L, A = setup()
    k, n = 65537, 65536
    dw, one = torch.full((k, n), 99.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, device="cuda")
    L.linear_bwd(L.linear_desc(0, n, k, wgrad_dtype=A.BF16), ptr(one), ptr(one), ptr(one), None, None, ptr(dw), None, None, stream(torch))
    torch.cuda.synchronize()
    assert not any(bool(c.any()) for c in dw.split(4096))


def test_distillation_of_many_rows():
    """More than 2^26 rows of two classes: loss, statistics and gradient of each, the same as a row of its kind alone."""
    torch, L, A = setup()
    rows = (1 << 26) + 5
    z = torch.zeros(rows, 2, dtype=torch.bfloat16, device="cuda")
    z[:, 1] = (torch.arange(rows, device="cuda") % 7).to(torch.bfloat16)
    ids, t, weight = (torch.arange(rows, device="cuda") % 2).int(), torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    scale = 1 / 64

    def calls(z, ids, t, weight):
        r = z.shape[0]
        d = L.distill_desc(r, 2, 1, scale=scale)
        ws = space(torch, L.distill_workspace_bytes(d, A.DISTILL_FWD))
        loss, row, lse, dz = torch.full((1,), 9.0, device="cuda"), torch.full((r,), 9.0, device="cuda"), torch.full((r,), 9.0, device="cuda"), torch.full_like(z, 9.0)
        L.distill_fwd(d, ptr(z), ptr(t), ptr(ids), ptr(weight), ptr(loss), ptr(row), ptr(lse), ptr(ws), stream(torch))
        L.distill_loss_grad(d, ptr(z), ptr(t), ptr(ids), ptr(weight), ptr(loss), ptr(dz), ptr(ws), stream(torch))
        torch.cuda.synchronize()
        return loss.item(), row, lse, dz
    loss, row, lse, dz = calls(z, ids, t, weight)
    few = calls(z[:14].clone(), ids[:14].clone(), t[:14].clone(), weight[:14].clone())
    same(torch, row, lambda i, j: few[1][torch.arange(i, j, device="cuda") % 14], "row_loss")
    same(torch, lse, lambda i, j: few[2][torch.arange(i, j, device="cuda") % 14], "lse")
    for c in range(2):
        same(torch, dz[:, c], lambda i, j: few[3][torch.arange(i, j, device="cuda") % 14, c], "dz")
    want = scale * row.double().sum().item()
    assert abs(loss - want) <= 2.0 ** -23 * want
