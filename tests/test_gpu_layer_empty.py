"""Language-model layers on tensors without rows."""
import pytest

from test_gpu_dense_layers import ptr, setup, stream

pytestmark = pytest.mark.gpu


def test_no_rows_of_empty_tensors():
    """Empty tensors have null pointers: gradients that do not depend on rows are zeros, and so is the loss."""
    torch, L, A = setup()
    x, dy = torch.empty(0, 24, device="cuda", dtype=torch.bfloat16), torch.empty(0, 40, device="cuda", dtype=torch.bfloat16)
    w, dw, dw2 = torch.zeros(24, 40, device="cuda", dtype=torch.bfloat16), torch.full((24, 40), 9.0, device="cuda"), torch.full((24, 40), 9.0, device="cuda")
    db, loss = torch.full((40,), 9.0, device="cuda"), torch.full((1,), 9.0, device="cuda")
    assert x.data_ptr() == 0 and dy.data_ptr() == 0
    d = L.linear_desc(0, 40, 24, act=A.ACT_GELU)
    L.linear_fwd(d, ptr(x), ptr(w), None, None, ptr(dy), None, None, stream(torch))
    L.linear_bwd(d, ptr(dy), ptr(x), ptr(w), ptr(dy), ptr(x), ptr(dw), ptr(db), None, stream(torch))
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()
    g = L.gated_desc(0, 40, 24)
    dw.fill_(9.0)
    L.gated_fwd(g, ptr(x), ptr(w), ptr(w), ptr(dy), ptr(dy), ptr(dy), None, stream(torch))
    L.gated_bwd(g, ptr(dy), ptr(x), ptr(w), ptr(w), ptr(dy), ptr(dy), ptr(x), ptr(dw), ptr(dw2), None, stream(torch))
    e = L.distill_desc(0, 40, 3)
    L.distill_loss_grad(e, ptr(dy), ptr(dy), ptr(dy), ptr(dy), ptr(loss), ptr(dy), None, stream(torch))
    torch.cuda.synchronize()
    assert not dw.any() and not dw2.any() and loss.item() == 0.0
