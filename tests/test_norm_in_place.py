"""A norm's result in the place of both operands (no GPU: a call that is not refused says PVT_ECUDA for want of one)."""
import ctypes

import pytest
import torch

from paper_2405_14852_b200 import binding as B


def apply(ldx, ldr, rows=3, **results):
    n = B.pvt_norm(rows=rows, cols=100, kind=B.PVT_NORM_RMS, x=0x1000, ldx=ldx, residual=0x1000, ldr=ldr, weight=None, bias=None,
                   dtype=B.PVT_BF16, weight_dtype=B.PVT_F32, eps=1e-5, reserved_=0)
    args = dict(total=None, ldt=100, y=None, y_dtype=B.PVT_BF16, ldy=100)
    args.update(results)
    return B.lib().pvt_norm_apply(ctypes.byref(n), args["total"], args["ldt"], args["y"], args["y_dtype"], args["ldy"], None, None, None)


@pytest.mark.parametrize("result", [lambda ld: dict(total=0x1000, ldt=ld), lambda ld: dict(y=0x1000, ldy=ld)])
@pytest.mark.parametrize("ldx,ldr", [(100, 200), (200, 100)])
def test_rows_have_to_lie_as_those_of_both_operands_do(result, ldx, ldr):
    """x and the residual begin at one address and go on at different distances: a row of the result is another row of one of them."""
    for ld in (ldx, ldr):
        assert apply(ldx, ldr, **result(ld)) == B.PVT_EINVAL
    if not torch.cuda.is_available():  # (made-up addresses)
        assert apply(ldx, ldx, **result(ldx)) == B.PVT_ECUDA  # both the same matrix
        assert apply(ldx, ldr, rows=1, **result(ldx)) == B.PVT_ECUDA  # one row has no distance
