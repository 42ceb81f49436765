"""Verification of drafted tokens on the GPU against the rule in fp64: counts of drafts, vocabularies from one class on, borders of the drawn numbers, no share, tokens that are no class."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def rule(p, q, drafted, counts, u, v):
    """One request after the other; p: (requests, drafts + 1, classes)."""
    b, d = drafted.shape
    accepted, tokens = np.zeros(b, int), np.full((b, d + 1), -1)
    for i in range(b):
        n = d if counts is None else min(max(int(counts[i]), 0), d)
        at = 0
        while at < n:
            t = drafted[i, at]
            if not (0 <= t < p.shape[2] and u[i, at] * q[i, at, t] < p[i, at, t]):
                break
            tokens[i, at] = t
            at += 1
        accepted[i] = at
        share = p[i, at] - q[i, at] if at < n else p[i, at]
        share = np.where(share > 0, share, 0)
        if not share.sum() > 0:
            share = np.where(p[i, at] > 0, p[i, at], 0)
        if share.sum() > 0:
            run = np.cumsum(share)
            hit = np.flatnonzero((run > v[i] * run[-1]) & (share > 0))
            tokens[i, at] = hit[0] if len(hit) else np.flatnonzero(share)[-1]
    return accepted, tokens


def call(torch, L, p, q, drafted, counts, u, v, pad=0):
    b, d = drafted.shape
    c = p.shape[2]

    def rows(t):
        out = torch.full((t.shape[0] * t.shape[1], c + pad), float("inf"), device="cuda")
        out[:, :c] = torch.as_tensor(t, dtype=torch.float32).reshape(-1, c).cuda()
        return out
    args = [rows(p), rows(q) if d else None] + [torch.as_tensor(t, dtype=k).cuda().contiguous() if t is not None else None
                                                 for t, k in ((drafted, torch.int32), (counts, torch.int32), (u, torch.float32), (v, torch.float32))]
    desc = L.verify_desc(b, d, c, ldp=c + pad, ldq=c + pad)
    ws = torch.full((L.verify_workspace_bytes(desc) + 16,), 255, dtype=torch.uint8, device="cuda")
    accepted, tokens = torch.full((b,), 99, dtype=torch.int32, device="cuda"), torch.full((b, d + 1), 99, dtype=torch.int32, device="cuda")
    L.verify(desc, *(None if t is None else t.data_ptr() for t in args), accepted.data_ptr(), tokens.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return accepted.cpu().numpy(), tokens.cpu().numpy()


def make(seed, b, d, c, spread=0.5, agree=0.3):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((b, d + 1, c)) * spread

    def soft(t):
        e = np.exp(t - t.max(2, keepdims=True))
        return (e / e.sum(2, keepdims=True)).astype(np.float32)
    p, q = soft(z), soft(z[:, :d] + rng.standard_normal((b, d, c)) * agree) if d else np.zeros((b, 0, c), np.float32)
    drafted = np.array([[rng.choice(c, p=q[i, j].astype(float) / q[i, j].astype(float).sum()) for j in range(d)] for i in range(b)], int).reshape(b, d)
    return p, q, drafted, rng.integers(0, d + 1, b), rng.random((b, d), dtype=np.float32), rng.random(b, dtype=np.float32)


@pytest.mark.parametrize("b,d,c,pad", [(1, 0, 1, 0), (1, 1, 1, 0), (3, 2, 2, 1), (5, 4, 100, 0), (40, 3, 1023, 3), (2, 70, 1025, 0), (7, 5, 4097, 0), (1, 4, 32003, 5), (1, 8, 131073, 0),
                                       (600, 2, 130, 0), (16, 6, 20000, 4), (256, 3, 16384, 0), (257, 2, 16384, 0), (3, 2, 16385, 1), (9, 3, 8200, 2), (2, 1024, 1500, 0)])
def test_against_the_rule(b, d, c, pad):
    import torch
    import paper_1807_02037_amd as L
    for seed, counted in ((1, True), (2, False)):
        p, q, t, n, u, v = make(seed, b, d, c)
        n = n if counted else None
        want = rule(p.astype(float), q.astype(float), t, n, u.astype(float), v.astype(float))
        got = call(torch, L, p, q, t, n, u, v, pad)
        assert (got[0] == want[0]).all() and (got[1] == want[1]).all(), np.argwhere(got[1] != want[1])


@pytest.mark.parametrize("times", [1, 20])
def test_borders(times):                                           # many requests take two launches
    import torch
    import paper_1807_02037_amd as L
    nan, inf = float("nan"), float("inf")
    c = 2100
    p, q = np.zeros((14, 2, c), np.float32), np.zeros((14, 1, c), np.float32)
    t, u, v = np.zeros((14, 1), int), np.full((14, 1), 0.5, np.float32), np.zeros(14, np.float32)
    p[:, :, 5], p[:, :, 2050], q[:, 0, 5], q[:, 0, 2050] = 0.25, 0.75, 0.25, 0.75
    t[:] = 5
    p[0, 0, 5], q[0, 0, 5], u[0] = 0.25, 0.5, 0.5                  # u q = p: not accepted; p - q is above 0 at no class but none: from p
    u[1] = 0.0                                                     # u = 0: accepted where p has a share
    u[2], p[2, 0, 5] = 0.0, 0.0                                    # and not where it has none
    t[3], t[4] = -1, c                                             # no class
    u[5] = nan
    q[6, 0, 5] = nan                                               # a class whose q is NaN has no share, and its draft is not accepted
    q[6, 0, 2050] = 0.5
    u[7], v[7] = 1.0, 1.0                                          # v = 1: the last class with a share
    p[8] = 0.0                                                     # no class has one
    p[9, 1] = 0.0
    p[9, 1, 2099], v[9] = 1e-30, 0.999                             # the last class, all accepted
    p[10, :, 7], t[10] = nan, 5
    p[11, 1, 5], p[11, 1, 2050], v[11] = 0.5, 0.5, 0.5             # half of the whole: the running sum has to be above
    p[12, 1], v[12] = 1.0 / 4096, 0.0                              # the first class
    p[13, 1, 5], v[13] = -1.0, 0.0                                 # below 0: no share
    p, q, t, u, v = (np.tile(a, (times,) + (1,) * (a.ndim - 1)) for a in (p, q, t, u, v))
    want = rule(p.astype(float), q.astype(float), t, None, u.astype(float), v.astype(float))
    got = call(torch, L, p, q, t, None, u, v)
    assert (got[0] == want[0]).all() and (got[1] == want[1]).all(), (got, want)
    assert got[1][8, 0] == -1 and got[1][11].tolist() == [5, 2050] and got[1][12].tolist() == [5, 0] and got[1][13].tolist() == [5, 2050] and got[1][6].tolist() == [2050, -1]


def test_counts_outside_are_cut():
    import torch
    import paper_1807_02037_amd as L
    p, q, t, _, u, v = make(4, 6, 3, 50)
    n = np.array([-5, 0, 1, 3, 4, 1000])
    got = call(torch, L, p, q, t, n, u, v)
    want = rule(p.astype(float), q.astype(float), t, np.clip(n, 0, 3), u.astype(float), v.astype(float))
    assert (got[0] == want[0]).all() and (got[1] == want[1]).all()


def test_the_drawn_tokens_follow_the_target():
    """Drafts from q, verified: the first token of each request is distributed as p.  40000 requests over 6 classes: a share is off by 6 deviations once in 10^9."""
    import torch
    import paper_1807_02037_amd as L
    rng = np.random.default_rng(0)
    n, p0, q0 = 40000, np.array([0.3, 0.05, 0.25, 0.1, 0.1, 0.2]), np.array([0.1, 0.3, 0.2, 0.2, 0.15, 0.05])
    p, q = np.broadcast_to(p0, (n, 2, 6)).astype(np.float32), np.broadcast_to(q0, (n, 1, 6)).astype(np.float32)
    t = rng.choice(6, p=q0, size=(n, 1))
    got = call(torch, L, p, q, t, None, rng.random((n, 1), dtype=np.float32), rng.random(n, dtype=np.float32))[1][:, 0]
    share = np.bincount(got, minlength=6) / n
    assert (np.abs(share - p0) < 6 * np.sqrt(p0 * (1 - p0) / n)).all(), share


def test_graph():
    import torch
    import paper_1807_02037_amd as L
    p, q, t, n, u, v = make(9, 4, 3, 9000)
    dev = [torch.as_tensor(x).cuda().contiguous() for x in (p, q, t.astype(np.int32), n.astype(np.int32), u, v)]
    desc = L.verify_desc(4, 3, 9000)
    ws = torch.empty(L.verify_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    acc, tok = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, 4, dtype=torch.int32, device="cuda")

    def run():
        L.verify(desc, *(x.data_ptr() for x in dev), acc.data_ptr(), tok.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            run()
    for seed in range(3):
        new = make(seed, 4, 3, 9000)
        for a, b in zip(dev, new):
            a.copy_(torch.as_tensor(b).to(a.dtype))
        g.replay()
        torch.cuda.synchronize()
        want = rule(*(x.astype(float) if x.dtype.kind == "f" else x for x in new))
        assert (acc.cpu().numpy() == want[0]).all() and (tok.cpu().numpy() == want[1]).all()
