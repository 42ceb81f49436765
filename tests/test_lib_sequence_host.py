"""Refusals, workspace sizes and calls without rows of the sequence operators (no GPU: every refusal comes before anything is launched)."""
import pytest

import paper_1807_02037_amd as L
from paper_1807_02037_amd import abi as A

PTR = 1 << 20        # never dereferenced


def refused(call, *args, match):
    with pytest.raises(L.LmsError, match=match) as e:
        call(*args)
    assert e.value.status == A.EINVAL


def recur(**kw):
    return L.recur_desc(**{**dict(rows=200, channels=300, seqs=4), **kw})


BAD_RECUR = [(dict(rows=-1), "rows must be"), (dict(channels=0), "channels"), (dict(seqs=0), "sequences"), (dict(rows=(1 << 31) - 1), "rows"), (dict(channels=(1 << 26) + 1), "channels"),
             (dict(seqs=(1 << 30) + 1), "sequences"), (dict(act=5), "activation"), (dict(dtype=A.I32), "dtype"), (dict(ldx=299), "pitch"), (dict(ldy=299), "pitch"),
             (dict(ldy=(1 << 40) + 1), "pitch")]


@pytest.mark.parametrize("kw,match", BAD_RECUR)
def test_recur_descriptors(kw, match):
    d = recur(**kw)
    refused(L.recur_workspace_bytes, d, A.RECUR_FWD, match=match)
    refused(L.recur_kept_bytes, d, match=match)
    refused(L.recur_fwd, d, PTR, PTR, None, PTR, None, PTR, None, PTR, PTR, None, match=match)
    refused(L.recur_bwd, d, PTR, PTR, PTR, PTR, PTR, None, PTR, None, PTR, PTR, PTR, None, PTR, None, match=match)
    refused(L.recur_step, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match=match)


def test_recur_calls():
    d = recur()
    n = 4 * 300 * 4
    refused(L.recur_workspace_bytes, d, 2, match="unknown call")
    refused(L.recur_fwd, d, None, PTR, None, PTR, None, PTR, None, PTR, PTR, None, match="null argument")
    refused(L.recur_fwd, d, PTR, PTR, None, PTR, None, PTR, None, PTR, None, None, match="workspace of")
    refused(L.recur_fwd, d, PTR, PTR, None, PTR, None, PTR, None, PTR, PTR + 8, None, match="workspace is not aligned")
    refused(L.recur_fwd, d, PTR, PTR, None, PTR, None, PTR, None, PTR + 8, PTR, None, match="workspace is not aligned")
    refused(L.recur_fwd, recur(seqs=3), PTR, PTR, None, None, None, PTR, None, PTR, PTR, None, match="multiple of the sequences")
    refused(L.recur_fwd, d, PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, PTR, None, match="overlap")
    refused(L.recur_fwd, d, PTR, PTR, None, PTR, PTR + n - 4, PTR, PTR, PTR, PTR, None, match="overlap")
    refused(L.recur_fwd, d, PTR + 1, PTR, None, PTR, None, PTR, None, PTR, PTR, None, match="aligned")
    refused(L.recur_fwd, d, PTR, PTR, None, PTR + 2, None, PTR, None, PTR, PTR, None, match="aligned")
    refused(L.recur_fwd, recur(dtype=A.F32), PTR, PTR, PTR + 2, PTR, None, PTR, None, PTR, PTR, None, match="aligned")
    refused(L.recur_bwd, d, PTR, PTR, PTR, PTR, PTR, None, None, None, PTR, PTR, PTR, None, PTR, None, match="kept is needed")
    refused(L.recur_bwd, d, PTR, PTR, PTR, None, PTR, None, PTR, None, PTR, PTR, PTR, None, PTR, None, match="needs o")
    refused(L.recur_bwd, d, PTR, PTR, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, PTR + n - 4, PTR, None, match="overlap")
    refused(L.recur_bwd, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, None, match="overlap")
    refused(L.recur_bwd, d, PTR, PTR, PTR, PTR, PTR, None, PTR, None, PTR, PTR, PTR, None, None, None, match="workspace of")
    refused(L.recur_step, d, PTR, PTR, PTR, None, PTR, PTR, PTR, None, match="null argument")
    refused(L.recur_step, d, PTR, PTR, PTR, PTR, PTR, PTR + 4, PTR, None, match="apart")
    refused(L.recur_step, recur(rows=65537), PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match="65536 rows")
    L.recur_step(recur(rows=0), None, None, None, None, None, None, None, None)


def test_recur_sizes():
    assert L.recur_kept_bytes(recur(rows=32)) == 0 and L.recur_workspace_bytes(recur(rows=32), A.RECUR_FWD) == 0
    assert L.recur_kept_bytes(recur(rows=65)) >= 3 * 300 * 4
    small, large = (L.recur_workspace_bytes(recur(rows=r, channels=1000), A.RECUR_BWD) for r in (1000, 1000000))
    assert small < large < 1000000 * 1000 * 2 // 4
    # sizes of 64 bits
    assert L.recur_kept_bytes(recur(rows=1 << 30, channels=1 << 20)) > 1 << 45


def norm(**kw):
    return L.group_norm_desc(**{**dict(n=3, s=10, c=12, groups=4), **kw})


@pytest.mark.parametrize("kw,match", [(dict(n=-1), "samples"), (dict(s=0), "positions"), (dict(c=0), "channels"), (dict(groups=5), "multiple of the groups"), (dict(groups=0), "multiple"),
                                      (dict(n=1 << 20, s=1 << 12), "rows"), (dict(n=1 << 62, s=4), "rows"), (dict(c=(1 << 20) + 4), "channels"), (dict(act=-1), "activation"),
                                      (dict(dtype=A.I32), "dtype"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(ldx=11), "pitch"),
                                      (dict(ldy=-12), "pitch")])
def test_norm_descriptors(kw, match):
    d = norm(**kw)
    refused(L.group_norm_workspace_bytes, d, A.GROUP_NORM_FWD, match=match)
    refused(L.group_norm_fwd, d, PTR, None, None, PTR, PTR, PTR, PTR, None, match=match)
    refused(L.group_norm_bwd, d, PTR, PTR, None, None, PTR, PTR, PTR, None, None, PTR, None, match=match)


def test_norm_calls():
    d = norm()
    refused(L.group_norm_workspace_bytes, d, 2, match="unknown call")
    refused(L.group_norm_fwd, d, None, None, None, PTR, PTR, PTR, PTR, None, match="null argument")
    refused(L.group_norm_bwd, d, PTR, PTR, None, None, None, PTR, PTR, None, None, PTR, None, match="null argument")
    refused(L.group_norm_fwd, d, PTR, None, None, PTR, PTR, PTR, None, None, match="workspace")
    refused(L.group_norm_fwd, d, PTR, None, None, PTR, PTR, PTR, PTR + 8, None, match="workspace is not aligned")
    refused(L.group_norm_fwd, d, PTR + 1, None, None, PTR, PTR, PTR, PTR, None, match="aligned")
    refused(L.group_norm_fwd, d, PTR, PTR + 2, None, PTR, PTR, PTR, PTR, None, match="aligned")
    refused(L.group_norm_bwd, d, PTR, PTR, None, None, PTR, PTR, PTR, PTR + 1, None, PTR, None, match="aligned")
    assert L.group_norm_workspace_bytes(norm(n=0), A.GROUP_NORM_BWD) == 0


def q8(**kw):
    return L.linear_q8_desc(**{**dict(m=4, n=8, k=20), **kw})


@pytest.mark.parametrize("kw,match", [(dict(m=-1), "rows must be"), (dict(k=0), "widths"), (dict(n=0), "widths"), (dict(m=1 << 31), "rows"), (dict(k=(1 << 17) + 1), "inputs"),
                                      (dict(n=(1 << 30) + 1), "widths"), (dict(act=5), "activation"), (dict(dtype=A.I32), "dtype"), (dict(ldx=19), "pitch"), (dict(ldw=7), "pitch"),
                                      (dict(ldy=7), "pitch"), (dict(ldr=7), "pitch"), (dict(ldx=(1 << 40) + 1), "pitch")])
def test_q8_descriptors(kw, match):
    d = q8(**kw)
    refused(L.linear_q8_weight_bytes, d, match=match)
    refused(L.linear_q8_workspace_bytes, d, match=match)
    refused(L.linear_q8_weight, d, PTR, PTR, PTR, None, match=match)
    refused(L.linear_q8_rows, d, PTR, PTR, PTR, None, match=match)
    refused(L.linear_q8_product, d, PTR, PTR, PTR, PTR, None, None, PTR, PTR, None, match=match)
    refused(L.linear_q8_fwd, d, PTR, PTR, PTR, None, None, PTR, PTR, None, match=match)


def test_q8_calls():
    d = q8()
    assert L.linear_q8_weight_bytes(d) == 8 * 32
    refused(L.linear_q8_weight, d, None, PTR, PTR, None, match="null argument")
    refused(L.linear_q8_weight, d, PTR, PTR + 8, PTR, None, match="16 bytes")
    refused(L.linear_q8_weight, d, PTR + 1, PTR, PTR, None, match="aligned")
    refused(L.linear_q8_rows, d, PTR, PTR + 4, PTR, None, match="16 bytes")
    refused(L.linear_q8_fwd, d, None, PTR, PTR, None, None, PTR, PTR, None, match="null argument")
    refused(L.linear_q8_fwd, d, PTR, PTR + 1, PTR, None, None, PTR, PTR, None, match="16 bytes")
    refused(L.linear_q8_fwd, d, PTR, PTR, PTR, None, None, PTR, None, None, match="workspace")
    refused(L.linear_q8_fwd, d, PTR, PTR, PTR, PTR + 2, None, PTR, PTR, None, match="aligned")
    refused(L.linear_q8_fwd, q8(ldr=9), PTR, PTR, PTR, None, PTR, PTR, PTR, None, match="same pitch")
    refused(L.linear_q8_product, q8(ldr=9), PTR, PTR, PTR, PTR, None, PTR, PTR, PTR, None, match="same pitch")
    L.linear_q8_fwd(q8(m=0), None, PTR, PTR, None, None, None, None, None)
    L.linear_q8_rows(q8(m=0), None, None, None, None)
    L.linear_q8_product(q8(m=0), None, None, PTR, PTR, None, None, None, None, None)
    assert L.linear_q8_workspace_bytes(q8(m=0)) == 0


def verify(**kw):
    return L.verify_desc(**{**dict(requests=3, drafts=2, classes=50), **kw})


@pytest.mark.parametrize("kw,match", [(dict(requests=-1), "requests"), (dict(drafts=-1), "drafts"), (dict(classes=0), "classes"), (dict(requests=(1 << 20) + 1), "requests"),
                                      (dict(drafts=1025), "drafts"), (dict(classes=(1 << 30) + 1), "classes"), (dict(ldp=49), "pitch"), (dict(ldq=49), "pitch"), (dict(requests=1 << 20, classes=1 << 15), "requests times classes"),
                                      (dict(ldq=1 << 41), "pitch")])
def test_verify_descriptors(kw, match):
    d = verify(**kw)
    refused(L.verify_workspace_bytes, d, match=match)
    refused(L.verify, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match=match)


def test_verify_calls():
    d = verify()
    refused(L.verify, d, None, PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, None, match="null argument")
    refused(L.verify, d, PTR, None, PTR, None, PTR, PTR, PTR, PTR, PTR, None, match="drafts need")
    refused(L.verify, d, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, None, None, match="workspace")
    refused(L.verify, d, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, PTR + 8, None, match="workspace")
    refused(L.verify, d, PTR + 2, PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, None, match="aligned")
    L.verify(verify(requests=0), None, None, None, None, None, None, None, None, None, None)


@pytest.mark.parametrize("make,kw", [(recur, dict(rows=1 << 64)), (recur, dict(channels=(1 << 32) + 12)), (recur, dict(seqs=(1 << 32) + 4)), (norm, dict(c=(1 << 32) + 12)),
                                     (norm, dict(n=(1 << 64) + 3)), (q8, dict(k=(1 << 32) + 20)), (verify, dict(requests=(1 << 32) + 3)), (verify, dict(classes=1 << 32))])
def test_numbers_that_do_not_fit(make, kw):
    with pytest.raises(L.LmsError, match=next(iter(kw))) as e:
        make(**kw)
    assert e.value.status == A.EINVAL
