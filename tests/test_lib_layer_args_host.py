"""Arguments of the language-model layers at their edges, without a GPU: calls without rows take the null pointers that empty tensors have; numbers that a field of a
descriptor cannot hold are refused and not cut."""
import pytest

import paper_1807_02037_amd as L
from paper_1807_02037_amd import abi as A
from test_lib_layers_host import PTR, distill, gated, linear, refused


def test_no_rows_come_with_null_pointers():
    for act in (A.ACT_NONE, A.ACT_SILU):
        d = linear(m=0, act=act)
        L.linear_fwd(d, None, PTR, None, None, None, None, None, None)
        L.linear_bwd(d, None, None, PTR, None, None, None, None, None, None)
    g = gated(m=0)
    L.gated_fwd(g, None, PTR, PTR, None, None, None, None, None)
    L.gated_bwd(g, None, None, PTR, PTR, None, None, None, None, None, None, None)
    L.distill_bwd(distill(rows=0), None, None, None, None, None, None, None, None)


def test_what_does_not_depend_on_rows_is_still_needed():
    refused(L.linear_fwd, linear(m=0), None, None, None, None, None, None, None, None, match="null argument")
    refused(L.gated_fwd, gated(m=0), None, PTR, None, None, None, None, None, None, match="null argument")
    refused(L.gated_bwd, gated(m=0), None, None, PTR, PTR, None, None, None, PTR, None, None, None, match="both")
    refused(L.distill_loss_grad, distill(rows=0), None, None, None, None, None, None, None, None, match="null argument")


def test_with_rows_every_pointer_is_needed():
    refused(L.linear_fwd, linear(m=1), None, PTR, None, None, PTR, None, None, None, match="null argument")
    refused(L.linear_bwd, linear(m=1), None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match="null argument")
    refused(L.gated_bwd, gated(m=1), None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, match="null argument")
    refused(L.distill_bwd, distill(rows=1), None, PTR, PTR, None, PTR, PTR, None, None, match="null argument")


@pytest.mark.parametrize("make,kw", [(linear, dict(n=(1 << 32) + 8)), (linear, dict(k=(1 << 32) + 16)), (linear, dict(m=(1 << 64) + 4)), (linear, dict(act=1 << 32)),
                                     (linear, dict(ldx=1 << 64)), (gated, dict(f=(1 << 32) + 8)), (gated, dict(k=-(1 << 32) + 16)), (gated, dict(ldh=(1 << 64) + 8)),
                                     (distill, dict(rows=1 << 64)), (distill, dict(classes=(1 << 32) + 100)), (distill, dict(k=(1 << 32) + 5)),
                                     (distill, dict(ldz=1 << 64))])
def test_numbers_that_do_not_fit(make, kw):
    with pytest.raises(L.LmsError, match=next(iter(kw))) as e:
        make(**kw)
    assert e.value.status == A.EINVAL
