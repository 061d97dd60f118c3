"""The calls on norms reject bad arguments before anything is enqueued (no GPU: a call that launched anything would say PVT_ECUDA)."""
import ctypes
import math

import pytest

from paper_2405_14852_b200 import binding as B


def norm(**kw):
    base = dict(rows=3, cols=100, kind=B.PVT_NORM_LAYER, x=0x1000, ldx=100, residual=None, ldr=0, weight=0x2000, bias=0x3000,
                dtype=B.PVT_BF16, weight_dtype=B.PVT_F32, eps=1e-5, reserved_=0)
    base.update(kw)
    return B.pvt_norm(**base)


def apply(n, total=None, ldt=100, y=0x8000, y_dtype=B.PVT_F32, ldy=100, yq=None, stats=None):
    return B.lib().pvt_norm_apply(n, total, ldt, y, y_dtype, ldy, yq, stats, None)


def grad(n, stats=0x9000, dtype=B.PVT_F32, dy=0xa000, ldy=100, res=None, ldr=100, dx=0xb000, ldx=100, dw=None, db=None,
         dw_dtype=B.PVT_F32, ws=None, ws_bytes=0):
    return B.lib().pvt_norm_grad(n, stats, dtype, dy, ldy, res, ldr, dx, ldx, dw, db, dw_dtype, 0, ws, ws_bytes, None)


BAD = [dict(rows=0), dict(rows=-1), dict(rows=2 ** 31), dict(cols=0), dict(cols=-3), dict(cols=32769, ldx=40000), dict(kind=2), dict(kind=-1),
       dict(x=None), dict(x=0x1001), dict(ldx=99), dict(ldx=1 << 41), dict(dtype=3), dict(dtype=-1), dict(dtype=B.PVT_F32, x=0x1002),
       dict(weight=0x2002), dict(bias=0x3001), dict(weight_dtype=3), dict(weight_dtype=B.PVT_F16, bias=0x3001), dict(eps=0.0),
       dict(eps=-1e-5), dict(eps=math.nan), dict(eps=math.inf)]


@pytest.mark.parametrize("kw", BAD)
def test_norms_are_checked(kw):
    n, before = ctypes.byref(norm(**kw)), B.pvt_launch_count()
    assert apply(n, ldt=1 << 20, ldy=1 << 20) == B.PVT_EINVAL
    assert grad(n, ldy=1 << 20, ldx=1 << 20) == B.PVT_EINVAL
    assert B.pvt_launch_count() == before


@pytest.mark.parametrize("kw", [dict(residual=0x4001, ldr=100), dict(residual=0x4000, ldr=99)])
def test_residuals_are_checked(kw):
    assert apply(ctypes.byref(norm(**kw))) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(y=None), dict(y=0x8002), dict(y_dtype=3), dict(ldy=99), dict(total=0x8001), dict(total=0x9000, ldt=99),
                                dict(total=0x8000, y_dtype=B.PVT_BF16), dict(stats=0x9004), dict(y=0x1000), dict(y=0x1000, y_dtype=B.PVT_BF16, ldy=104),
                                dict(total=0x1000, ldt=101)])
def test_results_are_checked(kw):
    assert apply(ctypes.byref(norm()), **kw) == B.PVT_EINVAL
    assert apply(None) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(rows=2), dict(cols=96), dict(format=5), dict(codes=0x1008), dict(ld=40), dict(scales=None),
                                dict(tensor_scale=0x3000)])
def test_four_bit_results_are_checked(kw):
    base = dict(rows=3, cols=100, format=B.PVT_MX_E8M0_32, reserved_=0, ld=64, codes=0x1000, scales=0x2000, tensor_scale=None)
    base.update(kw)
    assert apply(ctypes.byref(norm()), y=None, yq=ctypes.byref(B.pvt_mx(**base))) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(stats=None), dict(stats=0x9004), dict(dtype=3), dict(dy=None), dict(dy=0xa002), dict(ldy=99), dict(dx=None),
                                dict(dx=0xb001), dict(ldx=99), dict(res=0xc002), dict(res=0xc000, ldr=99), dict(dx=0xa000, ldx=104),
                                dict(dx=0x1000), dict(dx=0xc000, res=0xc000, ldr=104), dict(dw=0xd002, ws=0x10000, ws_bytes=1 << 30),
                                dict(dw=0xd004, dw_dtype=B.PVT_F64, ws=0x10000, ws_bytes=1 << 30),
                                dict(dw=0xd000, dw_dtype=B.PVT_F16, ws=0x10000, ws_bytes=1 << 30),
                                dict(dw=0xd000, db=0xd000, ws=0x10000, ws_bytes=1 << 30), dict(db=0xd001, ws=0x10000, ws_bytes=1 << 30),
                                dict(dw=0xd000), dict(dw=0xd000, ws=0x10080, ws_bytes=1 << 30)])
def test_gradients_are_checked(kw):
    assert grad(ctypes.byref(norm()), **kw) == B.PVT_EINVAL
    assert grad(None) == B.PVT_EINVAL


def test_the_residual_is_part_of_x_in_the_backward_call():
    assert grad(ctypes.byref(norm(residual=0x4000, ldr=100))) == B.PVT_EINVAL


def test_workspaces():
    n = norm()
    need = B.lib().pvt_norm_workspace_bytes(ctypes.byref(n))
    assert need >= 2 * 4 * 100 and need % 256 == 0
    assert grad(ctypes.byref(n), dw=0xd000, ws=0x10000, ws_bytes=need - 1) == B.PVT_EWORKSPACE
    for kw in (dict(rows=0), dict(cols=0), dict(cols=32769), dict(rows=1 << 31)):
        assert B.lib().pvt_norm_workspace_bytes(ctypes.byref(norm(**kw))) == 0
    assert B.lib().pvt_norm_workspace_bytes(None) == 0
    # depends on the shape alone, not on what is described
    assert B.lib().pvt_norm_workspace_bytes(ctypes.byref(norm(x=None, kind=9))) == need
