"""Gated recurrence on the GPU against fp64: sequences of no, one and many positions, their borders at every place of a chunk, odd channels and pitches, both types, gradients, the
single-token form, what masked rows and other sequences hold, streams and graphs."""
import numpy as np
import pytest

import sequence_oracle as S
from layer_oracle import f64

pytestmark = pytest.mark.gpu

ODD = [0, 1, 0, 7, 63, 64, 65, 0, 0, 130, 2, 1, 200, 0]           # lengths, with rows before and behind
# channels, lengths (or rows, sequences of one length), act, dtype, pad
CASES = [(1, [1], None, "fp32", 0), (4, [0, 0], "silu", "bf16", 0), (5, [3, 0, 1], "none", "bf16", 3), (256, ODD, "silu", "bf16", 0), (257, ODD, "gelu", "fp32", 1),
         (40, ODD, "gelu_tanh", "bf16", 8), (513, [1] * 70, "relu", "bf16", 5), (64, (64, 64), "silu", "bf16", 0), (64, (256, 8), "silu", "fp32", 0), (130, (300, 3), "silu", "bf16", 2),
         (300, (1500, 1), "silu", "bf16", 0), (16, [700, 0, 3, 900], None, "bf16", 0), (260, (192, 3), None, "fp32", 0),
         # work-groups that walk along sequences: steps of 64 rows that end in them, begin and end with them, pairs of channels that overlap
         (8190, (3 * 100, 3), "silu", "bf16", 2), (24577, (129, 1), "gelu", "fp32", 0), (2050, (12 * 65, 12), "relu", "bf16", 0), (130, (100 * 192, 100), None, "bf16", 1),
         (256, (96 * 224, 96), "gelu_tanh", "fp32", 0),
         # few channels: several runs of rows in a wave, in one and in several chunks
         (1, [3000, 0, 5000, 1, 777], "silu", "bf16", 0), (2, [9001], None, "fp32", 0), (3, (4200, 6), "gelu", "bf16", 1), (16, (3 * 1300, 3), "relu", "fp32", 0), (33, (5000, 2), "silu", "bf16", 3),
         (100, ODD, "gelu_tanh", "fp32", 0), (128, ODD * 3, "silu", "bf16", 0), (64, [1] * 300 + [0] * 9 + [4] * 50, "none", "bf16", 0), (20, (50, 1), "silu", "bf16", 0), (7, [40], "silu", "fp32", 0),
         (600, [50], "silu", "bf16", 0), (16, (64 * 128, 64), "silu", "bf16", 0),
         # many sequences without rows, before, between and behind others; nothing but them
         (300, [0] * 2000 + [3] + [0] * 1500 + [70, 1, 1] + [0] * 700, "silu", "bf16", 0), (3, [2, 0, 0, 0, 500] + [0] * 3000 + [1], "gelu", "fp32", 1), (40, [0] * 1000, "silu", "bf16", 0),
         (260, (0, 700), "relu", "fp32", 0), (516, [5] + [0] * 600 + [64] * 3 + [0] * 65 + [129], None, "bf16", 0)]


def make(torch, seed, c, lengths, act, dtype, pad):
    gen = torch.Generator().manual_seed(seed)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    if isinstance(lengths, tuple):
        rows, seqs, offsets = lengths[0], lengths[1], None
    else:
        seqs = len(lengths)
        offsets = np.concatenate([[0], np.cumsum(lengths)]) + (3 if seed % 2 else 0)
        rows = int(offsets[-1]) + 5 * (seed % 3)
        offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    def mat(shift=0.0, scale=1.0):
        t = torch.full((rows, c + pad), float("nan"))
        t[:, :c] = torch.randn(rows, c, generator=gen) * scale + shift
        if offsets is not None:                                    # rows of no sequence
            t[:int(offsets[0])] = float("nan")
            t[int(offsets[-1]):] = float("inf")
        return t.to(kind).cuda()[:, :c]
    d = dict(x=mat(), g=mat(1.5, 2.0), o=mat() if act is not None else None, dy=mat(), offsets=offsets, rows=rows, seqs=seqs, kind=kind)
    d["h0"], d["dlast"] = (torch.randn(seqs, c, generator=gen).cuda() for _ in range(2))
    return d


def ptr(t):
    return None if t is None else t.data_ptr()


def call(torch, L, d, c, act, pad, h0=True, dlast=True, stream=None):
    A = L.abi
    acts = {None: A.ACT_NONE, "none": A.ACT_NONE, "relu": A.ACT_RELU, "silu": A.ACT_SILU, "gelu": A.ACT_GELU, "gelu_tanh": A.ACT_GELU_TANH}
    s = stream or torch.cuda.current_stream().cuda_stream
    desc = L.recur_desc(d["rows"], c, d["seqs"], act=acts[act], dtype=A.BF16 if d["kind"] == torch.bfloat16 else A.F32, ldx=c + pad, ldy=c + pad)
    kept = torch.full((L.recur_kept_bytes(desc) + 16,), 255, dtype=torch.uint8, device="cuda")
    ws = torch.full((max(L.recur_workspace_bytes(desc, w) for w in (A.RECUR_FWD, A.RECUR_BWD)) + 16,), 255, dtype=torch.uint8, device="cuda")
    out = {n: torch.full((d["rows"], c + pad), 777.0, dtype=d["kind"], device="cuda") for n in ("y", "dx", "dg", "do")}
    out["last"], out["dh0"] = (torch.full((d["seqs"], c), 777.0, device="cuda") for _ in range(2))
    if act is None:
        out["do"] = None
    h0, dl = d["h0"] if h0 else None, d["dlast"] if dlast else None
    L.recur_fwd(desc, ptr(d["x"]), ptr(d["g"]), ptr(d["o"]), ptr(d["offsets"]), ptr(h0), ptr(out["y"]), ptr(out["last"]), ptr(kept), ptr(ws), s)
    ws.fill_(255)
    L.recur_bwd(desc, ptr(d["dy"]), ptr(d["x"]), ptr(d["g"]), ptr(d["o"]), ptr(d["offsets"]), ptr(h0), ptr(kept), ptr(dl), ptr(out["dx"]), ptr(out["dg"]), ptr(out["do"]),
                ptr(out["dh0"]), ptr(ws), s)
    return out


def check(torch, d, out, want, c):
    for name, got in out.items():
        if got is None:
            continue
        value, bound = want[name]
        if name in ("last", "dh0"):
            off = np.abs(f64(got) - value)
            assert (off <= bound).all(), (name, np.argwhere(~(off <= bound))[0], off.max())
            continue
        assert bool((got[:, c:] == got.new_tensor(777.0)).all()), name             # nothing between the rows
        used = torch.from_numpy(want["used"])
        assert bool((got.cpu()[~used] == got.new_tensor(777.0).cpu()).all()), name # nor in rows of no sequence
        off = np.abs(f64(got[:, :c])[want["used"]] - value[want["used"]])
        b = bound[want["used"]]
        assert (off <= b).all(), (name, np.argwhere(~(off <= b))[0], off.max())


def oracle(d, act, h0=True, dlast=True):
    zero = np.zeros(d["h0"].shape)
    with np.errstate(all="ignore"):
        return S.recur(f64(d["x"]), f64(d["g"]), None if d["o"] is None else f64(d["o"]), act or "none",
                       S.spans(d["rows"], d["seqs"], None if d["offsets"] is None else d["offsets"].cpu().numpy()), f64(d["h0"]) if h0 else zero, f64(d["dy"]),
                       f64(d["dlast"]) if dlast else zero, d["kind"])


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_fp64(i):
    import torch
    import paper_1807_02037_amd as L
    c, lengths, act, dtype, pad = CASES[i]
    d = make(torch, i, *CASES[i])
    states = i % 4 != 3
    out = call(torch, L, d, c, act, pad, states, states)
    torch.cuda.synchronize()
    check(torch, d, out, oracle(d, act, states, states), c)
    again = call(torch, L, d, c, act, pad, states, states)
    torch.cuda.synchronize()
    for k, v in out.items():
        assert v is None or torch.equal(v, again[k]), k            # the same bits


def test_gradients_against_differences():
    import torch
    rng = np.random.default_rng(5)
    rows, c = 9, 3
    x, g, o, dy = (rng.standard_normal((rows, c)) for _ in range(4))
    h0, dlast = rng.standard_normal((2, c)), rng.standard_normal((2, c))
    borders = [(0, 4), (4, 9)]

    def loss(x, g, o, h0):
        r = S.recur(x, g, o, "silu", borders, h0)
        return (r["y"][0] * dy).sum() + (r["last"][0] * dlast).sum()
    want = S.recur(x, g, o, "silu", borders, h0, dy, dlast)
    args = {"dx": x, "dg": g, "do": o, "dh0": h0}
    for name, t in args.items():
        for i in np.ndindex(t.shape):
            t0, step = t[i], 1e-5
            t[i] = t0 + step
            up = loss(x, g, o, h0)
            t[i] = t0 - step
            down = loss(x, g, o, h0)
            t[i] = t0
            assert abs((up - down) / (2 * step) - want[name][0][i]) < 1e-7, (name, i)


def test_gates_at_their_ends():
    """Gates that keep or replace all, and beyond where the exponential ends."""
    import torch
    import paper_1807_02037_amd as L
    d = make(torch, 1, 8, (96, 1), None, "fp32", 0)
    d["g"][:, 0], d["g"][:, 1], d["g"][:, 2], d["g"][:, 3], d["g"][:, 4] = 200.0, -200.0, 12.0, -12.0, 30.0
    d["g"][:, 5], d["g"][::2, 6], d["g"][1::2, 6] = -80.0, 95.0, -95.0
    out = call(torch, L, d, 8, None, 0)
    torch.cuda.synchronize()
    check(torch, d, out, oracle(d, None), 8)
    d["g"][:, 0], d["g"][:, 1] = float("inf"), float("-inf")
    out = call(torch, L, d, 8, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(out["last"][0, 0], d["h0"][0, 0]) and torch.equal(out["y"][:, 1], d["x"][:, 1])
    assert not out["dx"][:, 0].any() and torch.equal(out["dx"][:, 1], d["dy"][:, 1] + torch.nn.functional.one_hot(torch.tensor([95] * 96), 96)[0].cuda() * d["dlast"][0, 1])


@pytest.mark.parametrize("c", [12, 300])
def test_a_sequence_keeps_its_nan_to_itself(c):
    import torch
    import paper_1807_02037_amd as L
    lengths = [70, 5, 64, 3, 200, 9]
    d = make(torch, 2, c, lengths, "silu", "fp32", 0)
    clean = call(torch, L, d, c, "silu", 0)
    bad = dict(d)
    bad["x"], bad["dy"], bad["g"] = d["x"].clone(), d["dy"].clone(), d["g"].clone()
    off = [0] + list(np.cumsum(lengths))
    for s in (0, 2, 4):
        bad["x"][off[s]] = float("nan")
        bad["g"][off[s] + 1] = float("nan")
        bad["dy"][off[s + 1] - 1] = float("nan")
    got = call(torch, L, bad, c, "silu", 0)
    torch.cuda.synchronize()
    for s in (1, 3, 5):
        for n in ("y", "dx", "dg", "do"):
            assert torch.equal(got[n][off[s]:off[s + 1]], clean[n][off[s]:off[s + 1]]), (s, n)
        assert torch.equal(got["last"][s], clean["last"][s]) and torch.equal(got["dh0"][s], clean["dh0"][s])
    assert got["last"][0].isnan().all() and got["dh0"][4].isnan().all()


@pytest.mark.parametrize("packed", [True, False])
def test_long_sequences(packed):
    """The oracle on a few channels."""
    import torch
    import paper_1807_02037_amd as L
    c, rows = 1024, 40000
    d = make(torch, 8, c, [17000, 1, 22999] if packed else (rows, 2), "silu", "bf16", 0)
    out = call(torch, L, d, c, "silu", 0)
    torch.cuda.synchronize()
    few = [0, 255, 256, 700, 1023]
    part = {k: v[:, few] if torch.is_tensor(v) and v.dim() == 2 else v for k, v in d.items()}
    got = {k: v[:, few] for k, v in out.items()}
    check(torch, part, got, oracle(part, "silu"), len(few))


def test_a_line_in_several_launches():
    """More rows than a grid has work-groups for (2^21 of 64 rows, of 32 backward): the sequences on either side of the launches' borders against the same ones alone."""
    import torch
    import paper_1807_02037_amd as L
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows, border = (1 << 27) + 5000, [0, (1 << 26) - 700, (1 << 26) + 900, (1 << 27) - 333, (1 << 27) + 444, (1 << 27) + 5000]
    offsets = torch.tensor(border, dtype=torch.int32, device="cuda")
    d = dict(rows=rows, seqs=5, kind=torch.bfloat16, offsets=offsets)
    for n in ("x", "g", "o", "dy"):
        d[n] = torch.randn(rows, 1, generator=gen, device="cuda", dtype=torch.bfloat16)
    d["h0"], d["dlast"] = (torch.randn(5, 1, generator=gen, device="cuda") for _ in range(2))
    out = call(torch, L, d, 1, "silu", 0)
    for s in (1, 3, 4):
        b, e = border[s], border[s + 1]
        one = dict(d, rows=e - b, seqs=1, offsets=None, h0=d["h0"][s:s + 1], dlast=d["dlast"][s:s + 1], **{n: d[n][b:e].contiguous() for n in ("x", "g", "o", "dy")})
        got = {n: out[n][b:e] if n in ("y", "dx", "dg", "do") else out[n][s:s + 1] for n in out}
        check(torch, one, got, oracle(one, "silu"), 1)


@pytest.mark.parametrize("dtype,c,n,slots", [("bf16", 256, 5, 9), ("fp32", 1033, 3, 3), ("bf16", 4100, 70, 200), ("bf16", 3, 1, 1), ("bf16", 20, 1300, 40), ("fp32", 5, 2000, 1990)])
def test_step(dtype, c, n, slots):
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    gen = torch.Generator().manual_seed(n)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, g, o = (torch.randn(n, c + 3, generator=gen).to(kind).cuda()[:, :c] for _ in range(3))
    state = torch.randn(slots, c, generator=gen).cuda()
    ids = (torch.randperm(slots, generator=gen)[:n] if n <= slots else torch.randint(slots, (n,), generator=gen)).int()      # more rows than slots: positions far apart
    if n > 2:
        ids[1] = -1
    if n > 60:
        ids[5], ids[69], ids[68], ids[2] = ids[66], ids[66], slots, ids[66]        # one request's positions 2, 5, 66, 69; a slot that is not there
    desc = L.recur_desc(n, c, slots, act=A.ACT_SILU, dtype=A.BF16 if dtype == "bf16" else A.F32, ldx=c + 3, ldy=c)
    s = torch.cuda.current_stream().cuda_stream
    y, nxt = torch.full((n, c), 777.0, dtype=kind, device="cuda"), torch.full((slots, c), 777.0, device="cuda")
    L.recur_step(desc, x.data_ptr(), g.data_ptr(), o.data_ptr(), ids.cuda().data_ptr(), state.data_ptr(), nxt.data_ptr(), y.data_ptr(), s)
    place, y2 = state.clone(), torch.full_like(y, 777.0)
    dev = ids.cuda()
    L.recur_step(desc, x.data_ptr(), g.data_ptr(), o.data_ptr(), dev.data_ptr(), place.data_ptr(), place.data_ptr(), y2.data_ptr(), s)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    by_slot = {}
    for i, v in enumerate(ids.tolist()):
        if 0 <= v < slots:
            by_slot.setdefault(v, []).append(i)
    xx, gg, oo = f64(x), f64(g), f64(o)
    for v, idx in by_slot.items():
        want = S.recur(xx[idx], gg[idx], oo[idx], "silu", [(0, len(idx))], f64(state[v:v + 1]), dtype=kind)
        assert (np.abs(f64(y[idx]) - want["y"][0]) <= want["y"][1]).all()
        assert (np.abs(f64(nxt[v:v + 1]) - want["last"][0]) <= want["last"][1]).all()
        assert torch.equal(nxt[v], place[v])
    others = [v for v in range(slots) if v not in by_slot]
    assert bool((nxt[others] == 777.0).all()) and torch.equal(place[others], state[others])
    left = [i for i, v in enumerate(ids.tolist()) if not 0 <= v < slots]
    assert bool((y[left] == y.new_tensor(777.0)).all())


def test_steps_are_the_sequence():
    """A sequence token by token, and as one run."""
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    d = make(torch, 3, 96, (20, 1), "silu", "fp32", 0)
    out = call(torch, L, d, 96, "silu", 0)
    state, desc = d["h0"].clone(), L.recur_desc(1, 96, 1, act=A.ACT_SILU, dtype=A.F32)
    slot, y, s = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(20, 96, device="cuda"), torch.cuda.current_stream().cuda_stream
    for t in range(20):
        L.recur_step(desc, *(d[n][t].data_ptr() for n in ("x", "g", "o")), slot.data_ptr(), state.data_ptr(), state.data_ptr(), y[t].data_ptr(), s)
    torch.cuda.synchronize()
    want = oracle(d, "silu")
    check(torch, d, {"y": y, "last": state}, want, 96)
    check(torch, d, {"y": out["y"], "last": out["last"]}, want, 96)


def test_streams_and_graphs():
    """Two captured graphs with workspaces of their own, replayed with eager calls between; every replay against the eager result."""
    import torch
    import paper_1807_02037_amd as L
    ds = [make(torch, s, 256, ODD, "silu", "bf16", 0) for s in (6, 12)]
    eager = [call(torch, L, d, 256, "silu", 0) for d in ds]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for d in ds:
        with torch.cuda.stream(side):
            call(torch, L, d, 256, "silu", 0)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(call(torch, L, d, 256, "silu", 0))
            graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        call(torch, L, ds[0], 256, "silu", 0)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            for k in a:
                assert torch.equal(a[k], b[k]), k
                a[k].fill_(777.0)
        torch.cuda.synchronize()


@pytest.mark.parametrize("c,lengths", [(300, ODD), (40, ODD), (130, (100 * 192, 100))])
def test_gradients_that_are_not_asked_for(c, lengths):
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    d = make(torch, 6, c, lengths, "silu", "bf16", 0)
    full = call(torch, L, d, c, "silu", 0)
    s = torch.cuda.current_stream().cuda_stream
    desc = L.recur_desc(d["rows"], c, d["seqs"], act=A.ACT_SILU)
    kept = torch.empty(L.recur_kept_bytes(desc) + 16, dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(L.recur_workspace_bytes(desc, w) for w in (0, 1)) + 16, dtype=torch.uint8, device="cuda")
    y = torch.full_like(full["y"], 777.0)
    L.recur_fwd(desc, ptr(d["x"]), ptr(d["g"]), ptr(d["o"]), ptr(d["offsets"]), ptr(d["h0"]), ptr(y), None, None, ptr(ws), s)
    assert torch.equal(y, full["y"])                               # without the last states, nothing kept
    L.recur_fwd(desc, ptr(d["x"]), ptr(d["g"]), ptr(d["o"]), ptr(d["offsets"]), ptr(d["h0"]), ptr(y), None, ptr(kept), ptr(ws), s)
    for name in ("dx", "dg", "do", "dh0"):
        got = {name: torch.full_like(full[name], 777.0)}
        L.recur_bwd(desc, ptr(d["dy"]), ptr(d["x"]), ptr(d["g"]), ptr(d["o"]), ptr(d["offsets"]), ptr(d["h0"]), ptr(kept), ptr(d["dlast"]),
                    *(ptr(got.get(n)) for n in ("dx", "dg", "do", "dh0")), ptr(ws), s)
        assert torch.equal(got[name], full[name]), name
