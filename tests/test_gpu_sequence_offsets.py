"""Row pitches of 2^30 elements and more: offsets of the fifth row are beyond 32 bits, in elements and in bytes.  Results equal those of dense rows bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

PITCH, ROWS = (1 << 30) + 72, 5


def wide(torch, t, at):
    """The rows of t far apart, in a buffer of which nothing else is touched."""
    buf = torch.empty(ROWS * PITCH, dtype=t.dtype, device="cuda")
    out = buf.as_strided(t.shape, (PITCH, 1), at)
    out.copy_(t)
    return out


def test_recur_and_norm():
    import torch
    import paper_1807_02037_amd as L
    A = L.abi
    gen = torch.Generator(device="cuda").manual_seed(2)
    c, s = 64, torch.cuda.current_stream().cuda_stream

    def rand():
        return torch.randn(ROWS, c, generator=gen, device="cuda").bfloat16()
    x, g, dy, gamma = rand(), rand(), rand(), torch.randn(c, generator=gen, device="cuda")
    far = [wide(torch, t, 8) for t in (x, g, dy)]
    out_far = torch.empty(ROWS * PITCH, dtype=torch.bfloat16, device="cuda").as_strided((ROWS, c), (PITCH, 1), 8)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    y = torch.empty_like(x)
    for seqs in (1, 5):
        for ld, (xx, gg, _), out in ((0, (x, g, dy), y), (PITCH, far, out_far)):
            L.recur_fwd(L.recur_desc(ROWS, c, seqs, ldx=ld, ldy=ld), xx.data_ptr(), gg.data_ptr(), None, None, None, out.data_ptr(), None, None, ws.data_ptr(), s)
        assert torch.equal(y, out_far)
        for ld, (xx, gg, dd), out in ((0, (x, g, dy), y), (PITCH, far, out_far)):
            L.recur_bwd(L.recur_desc(ROWS, c, seqs, ldx=ld, ldy=ld), dd.data_ptr(), xx.data_ptr(), gg.data_ptr(), None, None, None, None, None, None, out.data_ptr(), None, None,
                        ws.data_ptr(), s)
        assert torch.equal(y, out_far)
    for n, sp, groups in ((ROWS, 1, 4), (1, ROWS, 4), (1, ROWS, 16), (ROWS, 1, 16)):
        mean, rstd = torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda")
        for ld, (xx, _, dd), out in ((0, (x, g, dy), y), (PITCH, far, out_far)):
            L.group_norm_fwd(L.group_norm_desc(n, sp, c, groups, ldx=ld, ldy=ld), xx.data_ptr(), gamma.data_ptr(), None, out.data_ptr(), mean.data_ptr(), rstd.data_ptr(), ws.data_ptr(), s)
        assert torch.equal(y, out_far)
        for ld, (xx, _, dd), out in ((0, (x, g, dy), y), (PITCH, far, out_far)):
            L.group_norm_bwd(L.group_norm_desc(n, sp, c, groups, ldx=ld, ldy=ld), dd.data_ptr(), xx.data_ptr(), gamma.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(), out.data_ptr(),
                             None, None, ws.data_ptr(), s)
        assert torch.equal(y, out_far)
    for rows in (1, ROWS):
        d = [L.linear_q8_desc(rows, c, c, act=A.ACT_SILU, ldx=ld, ldy=ld, ldr=ld) for ld in (0, PITCH)]
        wq, sw = torch.empty(L.linear_q8_weight_bytes(d[0]), dtype=torch.int8, device="cuda"), torch.empty(c, device="cuda")
        w = torch.randn(c, c, generator=gen, device="cuda").bfloat16()
        L.linear_q8_weight(d[0], w.data_ptr(), wq.data_ptr(), sw.data_ptr(), s)
        for desc, (xx, gg, _), out in zip(d, ((x, g, dy), far), (y, out_far)):
            L.linear_q8_fwd(desc, xx.data_ptr(), wq.data_ptr(), sw.data_ptr(), None, gg.data_ptr(), out.data_ptr(), ws.data_ptr(), s)
        assert torch.equal(y[:rows], out_far[:rows])


def test_verify():
    import torch
    import paper_1807_02037_amd as L
    gen = torch.Generator(device="cuda").manual_seed(2)
    c, d, pitch = 3000, 3, (1 << 30) + 72                          # fp32: the fourth row of p begins 12 GiB on
    p, q = (torch.softmax(torch.randn(n, c, generator=gen, device="cuda"), 1) for n in (d + 1, d))
    t, u, v = torch.randint(c, (1, d), device="cuda").int(), torch.zeros(1, d, device="cuda"), torch.full((1,), 0.7, device="cuda")
    far = []
    for m in (p, q):
        buf = torch.empty(m.shape[0] * pitch, device="cuda").as_strided(m.shape, (pitch, 1))
        buf.copy_(m)
        far.append(buf)
    out = []
    for ld, (a, b) in ((0, (p, q)), (pitch, far)):
        desc = L.verify_desc(1, d, c, ldp=ld, ldq=ld)
        ws = torch.empty(L.verify_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        acc, tok = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, d + 1, dtype=torch.int32, device="cuda")
        L.verify(desc, a.data_ptr(), b.data_ptr(), t.data_ptr(), None, u.data_ptr(), v.data_ptr(), acc.data_ptr(), tok.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
        out.append((acc.item(), tok.tolist()))
    assert out[0] == out[1] and out[0][0] == d                     # u = 0: all accepted, the token from the last row
