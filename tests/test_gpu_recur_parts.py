"""The recurrence's line in several launches, which only tensors of tens of gigabytes need: few chunks a launch are asked for instead.  Against fp64; and one call of
the real size."""
import numpy as np
import pytest

import test_gpu_recur as R

pytestmark = pytest.mark.gpu

# channels, lengths, act, dtype, pad, chunks a launch.  A chunk is 64 rows forward and 32 backward, times the runs of a wave where rows are narrow.
CASES = [
    # few chunks, which take what enters them from the sums where they are in one launch: sequences that cross the launches' borders
    (300, [500, 0, 60], "silu", "bf16", 0, 4), (257, [300, 1, 2], None, "fp32", 1, 5), (260, [1, 250], "gelu", "fp32", 0, 1),
    # more than 16 chunks both ways
    (300, [0, 700, 900, 3, 0, 600], "silu", "bf16", 2, 7), (513, [2200], "relu", "fp32", 0, 20), (256, [40] * 60 + [0] * 500 + [1200], None, "bf16", 0, 9),
    # few channels
    (40, [0, 800, 0, 0, 700, 5], "silu", "bf16", 0, 2), (3, [9000, 7000], "gelu_tanh", "fp32", 1, 1), (128, [3000, 0, 1100], None, "bf16", 0, 6), (16, [30000, 1, 9], "silu", "fp32", 0, 7)]


def launches(torch, call):
    """Kernels of the recurrence by name, and how often each was launched."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    out = {}
    for e in prof.key_averages():
        if "recur" in e.key:
            name = "join" if "join" in e.key else "line"
            out[name] = out.get(name, 0) + e.count
    return out


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_fp64(i, monkeypatch):
    import torch
    import paper_1807_02037_amd as L
    c, lengths, act, dtype, pad, part = CASES[i]
    d = R.make(torch, 20 + i, c, lengths, act, dtype, pad)
    monkeypatch.setenv("LMS_RECUR_CHUNKS", str(part))
    out = R.call(torch, L, d, c, act, pad)
    torch.cuda.synchronize()
    R.check(torch, d, out, R.oracle(d, act), c)
    # launches of sums, of what joins them (but for few chunks in one part) and of results for each part, forward and backward
    runs = 64 // min(64, 1 << (-(-c // 4) - 1).bit_length())
    chunks = [-(-d["rows"] // (rows * runs)) for rows in (64, 32)]
    parts = [-(-n // part) for n in chunks]
    assert max(parts) > 1
    assert launches(torch, lambda: R.call(torch, L, d, c, act, pad)) == {"join": sum(n for n, k in zip(parts, chunks) if n > 1 or k > 16), "line": 2 * sum(parts)}


def test_gradients_that_are_not_asked_for(monkeypatch):
    monkeypatch.setenv("LMS_RECUR_CHUNKS", "3")
    R.test_gradients_that_are_not_asked_for(300, [200, 0, 300, 77])


@pytest.mark.parametrize("c", [12, 300])
def test_a_sequence_keeps_its_nan_to_itself(c, monkeypatch):
    monkeypatch.setenv("LMS_RECUR_CHUNKS", "2")
    R.test_a_sequence_keeps_its_nan_to_itself(c)


def test_the_widest_line():
    """Nine chunks of 2^26 channels, eight a launch.  x, g and dy are one tensor; its gates are near 0.9975, so that the last row's gradient reaches the first."""
    import torch
    import paper_1807_02037_amd as L
    c, rows = 1 << 26, 257
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 48 GB of GPU memory")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, c, dtype=torch.bfloat16, device="cuda")
    wave = (torch.randn(rows, 1 << 16, generator=gen, device="cuda") * 0.3 + 6).bfloat16()
    x.view(rows, -1, 1 << 16).copy_(wave[:, None])
    desc = L.recur_desc(rows, c, 1)
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    kept = torch.zeros(L.recur_kept_bytes(desc), dtype=torch.uint8, device="cuda")             # h is in none of what is asked for
    ws = torch.empty(L.recur_workspace_bytes(desc, L.abi.RECUR_BWD), dtype=torch.uint8, device="cuda")
    dh0 = torch.full((1, c), 777.0, device="cuda")
    L.recur_bwd(desc, x.data_ptr(), x.data_ptr(), x.data_ptr(), None, offsets.data_ptr(), None, kept.data_ptr(), None, None, None, None, dh0.data_ptr(), ws.data_ptr(),
                torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    few = list(range(0, 1 << 16, 4099))
    w = R.f64(wave[:, few])
    zero = np.zeros((1, len(few)))
    value, bound = R.S.recur(w, w, None, "none", [(0, rows)], zero, w, zero)["dh0"]
    for at in (0, 1 << 25, c - (1 << 16)):
        assert (np.abs(R.f64(dh0[:, [at + i for i in few]]) - value) <= bound).all()
    assert torch.equal(dh0.view(-1, 1 << 16), dh0[:, :1 << 16].expand(c >> 16, -1))
