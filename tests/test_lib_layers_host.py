"""Refusals and workspace sizes of the linear layer, the gated projection and the distillation loss (no GPU: every refusal comes before anything is launched)."""
import pytest

import paper_1807_02037_amd as L
from paper_1807_02037_amd import abi as A

PTR = 1 << 20        # never dereferenced


def refused(call, *args, match):
    with pytest.raises(L.LmsError, match=match) as e:
        call(*args)
    assert e.value.status == A.EINVAL


def linear(**kw):
    return L.linear_desc(**{**dict(m=4, n=8, k=16), **kw})


def gated(**kw):
    return L.gated_desc(**{**dict(m=4, f=8, k=16), **kw})


def distill(**kw):
    return L.distill_desc(**{**dict(rows=4, classes=100, k=5), **kw})


BAD_SHAPES = [(dict(m=-1), "rows must be"), (dict(k=0), "widths"), (dict(m=1 << 31), "rows"), (dict(act=5), "activation"), (dict(act=-1), "activation"),
              (dict(dtype=A.I32), "dtype"), (dict(wgrad_dtype=A.I32), "wgrad_dtype"), (dict(dtype=A.F32, wgrad_dtype=A.BF16), "wgrad_dtype"),
              (dict(k=(1 << 30) + 1, ldx=0), "widths above"), (dict(ldx=15), "pitch"), (dict(ldw=7), "pitch"), (dict(ldx=-16), "pitch"), (dict(ldx=1 << 41), "pitch")]


@pytest.mark.parametrize("kw,match", BAD_SHAPES + [(dict(n=0), "widths"), (dict(ldy=7), "pitch"), (dict(ldr=1), "pitch")])
def test_linear_descriptors(kw, match):
    d = linear(**kw)
    refused(L.linear_workspace_bytes, d, A.LINEAR_FWD, match=match)
    refused(L.linear_fwd, d, PTR, PTR, None, None, PTR, None, PTR, None, match=match)
    refused(L.linear_bwd, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match=match)


@pytest.mark.parametrize("kw,match", BAD_SHAPES + [(dict(f=0), "widths"), (dict(ldh=7), "pitch")])
def test_gated_descriptors(kw, match):
    d = gated(**kw)
    refused(L.gated_workspace_bytes, d, A.GATED_FWD, match=match)
    refused(L.gated_fwd, d, PTR, PTR, PTR, PTR, None, None, PTR, None, match=match)
    refused(L.gated_bwd, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match=match)


@pytest.mark.parametrize("kw,match", [(dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(classes=(1 << 30) + 1), "classes"), (dict(classes=0), "classes"), (dict(k=0), "k must be"), (dict(k=1025), "k must be"),
                                      (dict(dtype=A.I32), "dtype"), (dict(ldz=99), "pitch"), (dict(ldz=-1), "pitch"), (dict(temperature=0.0), "temperature"),
                                      (dict(temperature=-1.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
                                      (dict(temperature=float("inf")), "temperature"), (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale")])
def test_distill_descriptors(kw, match):
    d = distill(**kw)
    refused(L.distill_workspace_bytes, d, A.DISTILL_FWD, match=match)
    refused(L.distill_fwd, d, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, None, match=match)
    refused(L.distill_bwd, d, PTR, PTR, PTR, None, PTR, PTR, PTR, None, match=match)
    refused(L.distill_loss_grad, d, PTR, PTR, PTR, None, PTR, PTR, PTR, None, match=match)


def test_null_pointers():
    for at in (0, 1, 4):
        args = [PTR, PTR, None, None, PTR, None, PTR, None]
        args[at] = None
        refused(L.linear_fwd, linear(), *args, match="null argument")
    refused(L.linear_bwd, linear(), None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match="null argument")
    refused(L.linear_bwd, linear(), PTR, PTR, None, PTR, PTR, None, None, PTR, None, match="dx needs w")
    refused(L.linear_bwd, linear(), PTR, None, PTR, PTR, None, PTR, None, PTR, None, match="dw needs x")
    refused(L.linear_bwd, linear(act=A.ACT_SILU), PTR, PTR, PTR, None, PTR, PTR, None, PTR, None, match="needs pre")
    for at in range(4):
        args = [PTR, PTR, PTR, PTR, None, None, PTR, None]
        args[at] = None
        refused(L.gated_fwd, gated(), *args, match="null argument")
    refused(L.gated_bwd, gated(), None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match="null argument")
    refused(L.gated_bwd, gated(), PTR, PTR, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, None, match="both")
    refused(L.gated_bwd, gated(), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, PTR, None, match="both")
    refused(L.gated_bwd, gated(), PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match="wg and wu are needed")
    refused(L.gated_bwd, gated(), PTR, None, PTR, PTR, None, None, PTR, None, None, PTR, None, match="x is needed")
    for at in (0, 1, 2):
        args = [PTR, PTR, PTR]
        args[at] = None
        refused(L.distill_fwd, distill(), *args, None, PTR, None, None, PTR, None, match="null argument")
    refused(L.distill_bwd, distill(), PTR, PTR, PTR, None, None, PTR, None, None, match="null argument")
    refused(L.distill_bwd, distill(), PTR, PTR, PTR, None, PTR, None, None, None, match="null argument")
    refused(L.distill_loss_grad, distill(), PTR, PTR, PTR, None, None, PTR, PTR, None, match="null argument")
    refused(L.distill_loss_grad, distill(), PTR, PTR, PTR, None, PTR, PTR, None, None, match="workspace of")
    with pytest.raises(L.LmsError, match="null argument"):
        A_ = A.lib()
        import ctypes as C
        b = C.c_uint64()
        from paper_1807_02037_amd.api import _ck
        _ck(A_.lms_linear_workspace_bytes(None, 0, C.byref(b)))


def test_alignment_of_elements():
    refused(L.linear_fwd, linear(), PTR + 1, PTR, None, None, PTR, None, PTR, None, match="aligned")
    refused(L.linear_fwd, linear(dtype=A.F32), PTR + 2, PTR, None, None, PTR, None, PTR, None, match="aligned")
    refused(L.linear_fwd, linear(), PTR, PTR, PTR + 2, None, PTR, None, PTR, None, match="aligned")
    refused(L.linear_bwd, linear(), PTR, PTR, PTR, None, PTR, PTR + 2, None, PTR, None, match="aligned")
    refused(L.gated_fwd, gated(), PTR, PTR, PTR + 1, PTR, None, None, PTR, None, match="aligned")
    refused(L.gated_bwd, gated(), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR + 2, PTR, PTR, None, match="aligned")
    refused(L.distill_fwd, distill(), PTR + 1, PTR, PTR, None, PTR, None, None, PTR, None, match="aligned")
    refused(L.distill_bwd, distill(), PTR, PTR + 2, PTR, None, PTR, PTR, None, None, match="aligned")


def test_residual_in_place_needs_its_pitch():
    refused(L.linear_fwd, linear(ldr=16), PTR, PTR, None, PTR, PTR, None, PTR, None, match="same pitch")


def test_missing_workspaces():
    d = linear(m=100, act=A.ACT_SILU)
    assert L.linear_workspace_bytes(d, A.LINEAR_BWD) >= 100 * 8 * 2
    refused(L.linear_bwd, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, None, match="workspace of")
    d = gated(m=100)
    assert L.gated_workspace_bytes(d, A.GATED_BWD) >= 2 * 100 * 8 * 2
    refused(L.gated_bwd, d, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, None, match="workspace of")
    refused(L.linear_bwd, linear(m=100), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR + 8, None, match="workspace is not aligned")
    refused(L.gated_bwd, gated(), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR + 4, None, match="workspace is not aligned")
    refused(L.distill_loss_grad, distill(), PTR, PTR, PTR, None, PTR, PTR, PTR + 4, None, match="workspace is not aligned")
    refused(L.linear_workspace_bytes, linear(), 2, match="unknown call")
    refused(L.gated_workspace_bytes, gated(), 3, match="unknown call")
    refused(L.distill_workspace_bytes, distill(), -1, match="unknown call")


def test_no_rows_need_nothing():
    """Calls without rows succeed where there is nothing to write."""
    L.linear_fwd(linear(m=0), PTR, PTR, None, None, PTR, None, None, None)
    L.gated_fwd(gated(m=0), PTR, PTR, PTR, PTR, None, None, None, None)
    assert L.distill_workspace_bytes(distill(rows=0), A.DISTILL_FWD) == 0
