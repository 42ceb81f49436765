"""Distillation loss and gradient on the GPU against fp64: vocabularies from one class on, odd ones, row pitches, rows without entries, masked classes, repeated
classes, both types."""
import math

import numpy as np
import pytest

import layer_oracle as O

pytestmark = pytest.mark.gpu

# rows, classes, k
SIZES = [(1, 1, 1), (3, 2, 2), (5, 17, 4), (2, 64, 64), (33, 100, 7), (9, 1000, 20), (4, 2049, 129), (3, 8191, 256), (2, 32003, 64), (3, 50304, 1024),
         (2, 131072, 33), (2, 160001, 8)]
U32 = 2.0 ** -24


def make(torch, seed, rows, classes, k, kind, pad):
    g = torch.Generator().manual_seed(seed)
    z = torch.full((rows, classes + pad), float("nan"))
    z[:, :classes] = torch.randn(rows, classes, generator=g) * 3
    ids = torch.randint(-1, classes, (rows, k), generator=g).int()                # repeated classes, and places without one
    t = torch.randn(rows, k, generator=g) * 3
    weight = torch.rand(rows, generator=g) + 0.5
    if rows > 2:
        ids[1] = -1                                                                # a row without entries
        weight[2] = 0
        t[0, 0] = -math.inf
        ids[0, -1] = classes                                                       # no such class: not there
    if classes > 50 and seed % 2:
        masked = torch.rand(classes, generator=g) < 0.2
        masked[ids[ids >= 0].long().clamp(max=classes - 1)] = False
        z[:, :classes][:, masked] = -math.inf
    return z.to(kind).cuda()[:, :classes], t.cuda(), ids.cuda(), weight.cuda()


def bounds(z, t, temp, scale, weight, classes, k):
    """Of lse, the row loss and dz in fp32.  x = z / T is rounded, and log2(e) times it once more: |x| 4 u in the argument of an exponential, which is off by as much
    relative to itself, and so are the sums, whose roundings add (classes + k) u at most."""
    x, v = np.abs(z / temp), np.abs(t / temp)
    big = np.where(np.isfinite(x), x, 0).max(1) + np.where(np.isfinite(v), v, 0).max(1) + 12
    e = U32 * (8 * big + 0.1 * classes + k + 16)
    # the running sum of a thread holds a few hundred terms at most and grows toward its total: a tenth of all terms bounds its roundings
    return e, temp * temp * e * 4, (scale * temp * weight)[:, None] * e[:, None] * 4


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_distill(i, dtype):
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    rows, classes, k = SIZES[i]
    kind, code = (torch.bfloat16, A.BF16) if dtype == "bf16" else (torch.float32, A.F32)
    temp, pad = (1.0, 2.0, 0.5)[i % 3], (0, 8, 5)[i % 3]
    scale = 1.0 / rows
    z, t, ids, weight = make(torch, i, rows, classes, k, kind, pad)
    s = torch.cuda.current_stream().cuda_stream
    d = L.distill_desc(rows, classes, k, temperature=temp, scale=scale, dtype=code, ldz=classes + pad)
    ws = torch.full((max(16, L.distill_workspace_bytes(d, A.DISTILL_FWD)),), 255, dtype=torch.uint8, device="cuda")
    loss, row_loss, lse = torch.full((1,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    dz = torch.full((rows, classes + pad), 777.0, dtype=kind, device="cuda")
    L.distill_fwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), loss.data_ptr(), row_loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), s)
    L.distill_bwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), lse.data_ptr(), dz.data_ptr(), None, s)
    torch.cuda.synchronize()
    zz, tt, ii, ww = O.f64(z), O.f64(t), ids.cpu().numpy(), O.f64(weight)
    want = O.distill(zz, tt, ii, ww, temp, scale)
    e_lse, e_row, e_dz = bounds(zz, tt, temp, scale, ww, classes, k)
    assert (np.abs(O.f64(lse) - want[2]) <= e_lse).all()
    assert (np.abs(O.f64(row_loss) - want[1]) <= e_row + U32 * np.abs(want[1])).all()
    assert abs(loss.item() - want[0]) <= scale * (ww * e_row).sum() + 4 * U32 * abs(want[0])
    off = np.abs(O.f64(dz[:, :classes]) - want[3])
    allowed = O.U[kind] * np.abs(want[3]) + e_dz
    assert (off <= allowed).all(), (np.argwhere(off > allowed)[0], off.max())
    assert bool((dz[:, classes:] == dz.new_tensor(777.0)).all())                   # nothing between the rows
    if rows > 2:
        assert not dz[1, :classes].any() and not dz[2, :classes].any() and row_loss[1] == 0
    # loss and gradient together, and in place
    both, loss2 = torch.full_like(dz, 777.0), torch.full((1,), 9.0, device="cuda")
    L.distill_loss_grad(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), loss2.data_ptr(), both.data_ptr(), ws.data_ptr(), s)
    torch.cuda.synchronize()
    assert torch.equal(loss2, loss)
    off = np.abs(O.f64(both[:, :classes]) - want[3])
    assert (off <= allowed).all(), (np.argwhere(off > allowed)[0], off.max())
    L.distill_loss_grad(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), loss2.data_ptr(), z.data_ptr(), ws.data_ptr(), s)
    torch.cuda.synchronize()
    assert torch.equal(loss2, loss) and torch.equal(z, both[:, :classes])


def test_without_weights_and_optional_outputs():
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    z, t, ids, _ = make(torch, 4, 12, 300, 6, torch.float32, 0)
    s = torch.cuda.current_stream().cuda_stream
    d = L.distill_desc(12, 300, 6, temperature=2.0, scale=0.25, dtype=A.F32)
    ws = torch.empty(L.distill_workspace_bytes(d, A.DISTILL_FWD), dtype=torch.uint8, device="cuda")
    ones, a, b, row = torch.ones(12, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(12, device="cuda")
    L.distill_fwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), None, a.data_ptr(), None, None, ws.data_ptr(), s)
    L.distill_fwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), ones.data_ptr(), b.data_ptr(), row.data_ptr(), None, ws.data_ptr(), s)
    assert torch.equal(a, b)
    only = torch.empty(12, device="cuda")
    L.distill_fwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), None, None, only.data_ptr(), None, None, s)
    assert torch.equal(only, row)
    # no rows: the loss is zero
    none = L.distill_desc(0, 300, 6, dtype=A.F32)
    L.distill_fwd(none, z.data_ptr(), t.data_ptr(), ids.data_ptr(), None, a.data_ptr(), None, None, None, s)
    assert a.item() == 0.0


def test_masks_that_leave_nothing():
    """All classes masked, or the teacher's class: infinite loss, finite gradient -p; the type's lowest value is an ordinary logit."""
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    for kind, code in ((torch.bfloat16, A.BF16), (torch.float32, A.F32)):
        z = torch.zeros(4, 70, device="cuda").to(kind)
        z[0] = -math.inf
        z[1, 5] = -math.inf
        z[2] = torch.finfo(kind).min
        z[3, 6:] = torch.finfo(kind).min
        t, ids = torch.zeros(4, 1, device="cuda"), torch.full((4, 1), 5, dtype=torch.int32, device="cuda")
        d = L.distill_desc(4, 70, 1, dtype=code)
        ws, row, lse, loss = torch.empty(256, dtype=torch.uint8, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty(1, device="cuda")
        dz = torch.empty_like(z)
        s = torch.cuda.current_stream().cuda_stream
        L.distill_fwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), None, loss.data_ptr(), row.data_ptr(), lse.data_ptr(), ws.data_ptr(), s)
        L.distill_bwd(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), None, lse.data_ptr(), dz.data_ptr(), None, s)
        torch.cuda.synchronize()
        assert row[0] == math.inf and row[1] == math.inf and loss.item() == math.inf
        assert torch.isfinite(dz.float()).all() and dz[0, 5] == -1 and not dz[0, :5].any() and dz[1, 5] == -1
        # 70 equal logits, and six of them
        assert lse[0] == -math.inf and abs(row[2].item() - math.log(70)) < 1e-5 and abs(row[3].item() - math.log(6)) < 1e-5
        step = torch.empty_like(z)
        L.distill_loss_grad(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), None, loss.data_ptr(), step.data_ptr(), ws.data_ptr(), s)
        torch.cuda.synchronize()
        # (in fp32 the logarithm of 70 is lost in lse beside 3e38, which the gradient from lse can do nothing about)
        assert abs(step[2, 0].float().item() - 1 / 70) < 1e-4 and torch.equal(step[0], dz[0]) and torch.equal(step[3], dz[3])
        assert not dz[3, 6:].any() and abs(dz[3, 0].float().item() - 1 / 6) < 1e-3


def test_gradient_is_the_slope_of_the_loss():
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    z, t, ids, weight = make(torch, 2, 20, 90, 9, torch.float32, 0)
    s = torch.cuda.current_stream().cuda_stream
    d = L.distill_desc(20, 90, 9, temperature=1.5, scale=1.0, dtype=A.F32)
    ws, loss, dz = torch.empty(256, dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    L.distill_loss_grad(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), loss.data_ptr(), dz.data_ptr(), ws.data_ptr(), s)
    step = 2.0 ** -5 / dz.norm().item()

    def at(shift):
        zz = (z + shift * dz).contiguous()
        L.distill_fwd(d, zz.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), loss.data_ptr(), None, None, ws.data_ptr(), s)
        return loss.item()
    slope = (at(step) - at(-step)) / (2 * step)
    want = dz.double().square().sum().item()
    assert abs(slope - want) <= 5e-3 * want, (slope, want)


def test_replays_of_a_captured_call():
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    z, t, ids, weight = make(torch, 6, 40, 3000, 16, torch.bfloat16, 0)
    d = L.distill_desc(40, 3000, 16, temperature=2.0, scale=0.1)
    ws = torch.empty(L.distill_workspace_bytes(d, A.DISTILL_LOSS_GRAD), dtype=torch.uint8, device="cuda")

    def call(loss, dz):
        L.distill_loss_grad(d, z.data_ptr(), t.data_ptr(), ids.data_ptr(), weight.data_ptr(), loss.data_ptr(), dz.data_ptr(), ws.data_ptr(),
                            torch.cuda.current_stream().cuda_stream)
    pairs = [(torch.empty(1, device="cuda"), torch.empty_like(z)) for _ in range(2)]
    call(*pairs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*pairs[1])
    for i in range(4):
        z.copy_(make(torch, 20 + 2 * i, 40, 3000, 16, torch.bfloat16, 0)[0])
        call(*pairs[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pairs[0][0], pairs[1][0]) and torch.equal(pairs[0][1], pairs[1][1]), i
