"""The gated recurrence with gates near their ends, as states of long memory have them: what a position takes in is (1 - a) x to its own precision, where a is 1 but for a few units of its last
place.  Every form: the line, wide and narrow, sequences that are walked along, single positions."""
import numpy as np
import pytest

import gate_oracle as G
import test_gpu_recur as R

pytestmark = pytest.mark.gpu

# gates: mean and spread
GATES = [(2.0, 1.0), (7.0, 1.0), (9.0, 1.0), (11.0, 1.0), (13.0, 1.0), (16.0, 1.0), (12.0, 0.0), (17.5, 0.0), (25.0, 3.0), (-9.0, 3.0), (0.0, 12.0)]
# channels, lengths, act, dtype, pad, and whether the states begin at 0
FORMS = {"line": (300, [500, 0, 73], "silu", "fp32", 0, True), "narrow": (5, [3000, 1, 40], None, "fp32", 1, True), "one chunk": (64, [50], "none", "fp32", 0, True),
         "line16": (300, [500, 0, 73], "silu", "bf16", 0, True), "states": (257, [400, 1], "gelu", "fp32", 0, False), "walk": (130, (100 * 192, 100), "silu", "fp32", 0, True),
         "walk16": (130, (100 * 192, 100), None, "bf16", 0, True)}


def oracle(d, act, zero):
    h0 = R.f64(d["h0"]) * (0 if zero else 1)
    with np.errstate(all="ignore"):
        return G.recur(R.f64(d["x"]), R.f64(d["g"]), None if d["o"] is None else R.f64(d["o"]), act or "none",
                       R.S.spans(d["rows"], d["seqs"], None if d["offsets"] is None else d["offsets"].cpu().numpy()), h0, R.f64(d["dy"]), R.f64(d["dlast"]), d["kind"])


@pytest.mark.parametrize("form,gate", [(f, g) for f in FORMS for g in GATES if "walk" not in f or g[0] in (2.0, 7.0, 13.0, 17.5, 0.0)])
def test_against_fp64(form, gate):
    import torch
    import paper_1807_02037_amd as L
    c, lengths, act, dtype, pad, zero = FORMS[form]
    d = R.make(torch, 32, c, lengths, act, dtype, pad)
    d["g"].copy_(torch.randn(d["g"].shape, generator=torch.Generator().manual_seed(1)) * gate[1] + gate[0])
    out = R.call(torch, L, d, c, act, pad, h0=not zero)
    torch.cuda.synchronize()
    R.check(torch, d, out, oracle(d, act, zero), c)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_single_positions(dtype):
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    n, c = 200, 9
    gen = torch.Generator().manual_seed(3)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, g = torch.randn(n, c, generator=gen).to(kind).cuda(), torch.linspace(-30, 30, n)[:, None].expand(n, c).to(kind).contiguous().cuda()
    for scale in (0.0, 1e-4, 1.0):
        state, y = torch.randn(n, c, generator=gen).cuda() * scale, torch.empty(n, c, dtype=kind, device="cuda")
        new, slots = state.clone(), torch.arange(n, dtype=torch.int32, device="cuda")
        desc = L.recur_desc(n, c, n, dtype=A.BF16 if dtype == "bf16" else A.F32)
        L.recur_step(desc, x.data_ptr(), g.data_ptr(), None, slots.data_ptr(), new.data_ptr(), new.data_ptr(), y.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        zero = np.zeros((n, c))
        want = G.recur(R.f64(x), R.f64(g), None, "none", [(i, i + 1) for i in range(n)], R.f64(state), zero, zero, kind)
        for got, (value, bound) in ((y, want["y"]), (new, want["last"])):
            off = np.abs(R.f64(got) - value)
            assert (off <= bound).all(), (scale, np.argwhere(~(off <= bound))[0], off.max())
