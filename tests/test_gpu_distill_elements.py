"""The distillation's gradient element by element, relative to the element's own probabilities, in every form that a row's length selects."""
import numpy as np
import pytest

import distill_bounds as B
import layer_oracle as O
from helpers import kernel_names

pytestmark = pytest.mark.gpu

# rows, classes, k; threads and vectors of the kernel in bf16 and in fp32
FORMS = [(5, 500, 7, (64, 1), (64, 1)), (4, 2001, 40, (64, 4), (64, 4)), (3, 8190, 64, (256, 4), (256, 4)), (3, 16383, 200, (512, 4), (512, 4)),
         (3, 32003, 64, (512, 8), (512, 8)), (2, 50304, 1024, (512, 13), (1024, 8)), (2, 65529, 33, (1024, 8), (1024, 8)), (2, 98299, 64, (1024, 12), (1024, 0)),
         (2, 131075, 129, (1024, 0), (1024, 0))]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(FORMS)))
def test_gradient_elements(i, dtype):
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    rows, classes, k, form, form32 = FORMS[i]
    kind, code = (torch.bfloat16, A.BF16) if dtype == "bf16" else (torch.float32, A.F32)
    pad, temp, scale = (0, 8, 3)[i % 3], (2.0, 1.0, 0.5)[i % 3], 0.5
    g = torch.Generator(device="cuda").manual_seed(i)
    full = torch.full((rows + 1, classes + pad), float("nan"), device="cuda")
    full[:rows, :classes] = torch.randn(rows, classes, generator=g, device="cuda") * 3
    full = full.to(kind)
    z = full[:rows, :classes]
    ids = torch.stack([torch.randperm(classes, generator=g, device="cuda")[:k] for _ in range(rows)]).int()
    ids[0, 0], ids[-1, -1] = classes - 1, 0                        # the row's ends
    if k > 8:
        ids[0, 3], ids[1, 5] = ids[0, 7], -1                       # a class twice, and a place without one
    t = torch.randn(rows, k, generator=g, device="cuda") * 3
    weight = torch.rand(rows, generator=g, device="cuda") + 0.5
    d = L.distill_desc(rows, classes, k, temperature=temp, scale=scale, dtype=code, ldz=classes + pad)
    ws = torch.full((L.distill_workspace_bytes(d, A.DISTILL_LOSS_GRAD),), 255, dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    dz = [torch.full_like(full, 777.0) for _ in range(2)]
    s = torch.cuda.current_stream().cuda_stream
    args = (z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr())

    def calls():
        L.distill_loss_grad(d, *args, loss.data_ptr(), dz[0].data_ptr(), ws.data_ptr(), s)
        L.distill_fwd(d, *args, None, None, lse.data_ptr(), None, s)
        L.distill_bwd(d, *args, lse.data_ptr(), dz[1].data_ptr(), None, s)
    names = kernel_names(calls)
    nt, nv = form if dtype == "bf16" else form32
    assert any(f"distill_kernel<{'unsigned short' if dtype == 'bf16' else 'float'}, {nt}, {nv}>" in v for v in names), names
    zz, tt, ii, ww = O.f64(z), O.f64(t), ids.cpu().numpy(), O.f64(weight)
    for got, from_lse in zip(dz, (False, True)):
        want, bound = B.gradient(zz, tt, ii, ww, temp, scale, O.U[kind], from_lse)
        off = np.abs(O.f64(got[:rows, :classes]) - want)
        assert (off <= bound).all(), (from_lse, int((off > bound).sum()), np.argwhere(off > bound)[0], (off / bound).max())
        assert bool((got[:, classes:] == 777).all()) and bool((got[rows:] == 777).all())
    both = dz[0].clone()
    L.distill_loss_grad(d, *args, loss.data_ptr(), z.data_ptr(), ws.data_ptr(), s)          # over the logits
    assert torch.equal(z, both[:rows, :classes])
