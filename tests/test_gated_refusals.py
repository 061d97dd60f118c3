"""The calls on gated products reject bad arguments before anything is enqueued (no GPU: a call that launched anything would say
PVT_ECUDA)."""
import ctypes

import pytest

from paper_2405_14852_b200 import binding as B

r = ctypes.byref


def mx(**kw):
    base = dict(rows=64, cols=256, format=B.PVT_MX_E8M0_32, reserved_=0, ld=128, codes=0x1000, scales=0x2000, tensor_scale=None)
    base.update(kw)
    return B.pvt_mx(**base)


def gated(x=None, wg=None, wu=None, act=0, h=0x8000, dtype=B.PVT_F32, ld=64, hq=None, status=None):
    return B.lib().pvt_mx_gated(r(x or mx(rows=5)), r(wg or mx()), r(wu or mx()), act, h, dtype, ld, hq and r(hq), status, None)


def grad(x=None, wg=None, wu=None, act=0, dh=0x8000, dtype=B.PVT_F32, ld=64, dgate=0x9000, dup=0xa000, ldd=64, status=None):
    return B.lib().pvt_mx_gated_grad(r(x or mx(rows=5)), r(wg or mx()), r(wu or mx()), act, dh, dtype, ld, dgate, dup, ldd, status, None)


def grad_input(dgate=0x9000, dup=0xa000, ldd=64, tokens=5, wg=None, wu=None, dx=0xb000, dtype=B.PVT_BF16, ld=256, status=None):
    return B.lib().pvt_mx_gated_grad_input(dgate, dup, ldd, tokens, r(wg or mx()), r(wu or mx()), dx, dtype, ld, status, None)


BAD_MX = [dict(rows=0), dict(cols=0), dict(format=2), dict(codes=None), dict(codes=0x1008), dict(scales=None), dict(scales=0x2004), dict(ld=120),
          dict(ld=112), dict(tensor_scale=0x3000), dict(format=B.PVT_MX_E4M3_16, tensor_scale=0x3002)]


@pytest.mark.parametrize("kw", BAD_MX)
def test_matrices_are_checked(kw):
    before = B.pvt_launch_count()
    for name in ("x", "wg", "wu"):
        assert gated(**{name: mx(**kw)}) == B.PVT_EINVAL and grad(**{name: mx(**kw)}) == B.PVT_EINVAL
        if name != "x":
            assert grad_input(**{name: mx(**kw)}) == B.PVT_EINVAL
    if kw != dict(ld=112):  # (enough for 64 columns)
        assert gated(hq=mx(**{**dict(rows=5, cols=64), **kw})) == B.PVT_EINVAL
    assert B.pvt_launch_count() == before


def test_null_matrices():
    lib, m = B.lib(), r(mx())
    assert lib.pvt_mx_gated(None, m, m, 0, 0x8000, 0, 64, None, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_gated(m, m, None, 0, 0x8000, 0, 64, None, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_gated_grad(m, None, m, 0, 0x8000, 0, 64, 0x9000, 0xa000, 64, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_gated_grad_input(0x9000, 0xa000, 64, 5, m, None, 0xb000, 0, 256, None, None) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(format=B.PVT_MX_E4M3_16), dict(cols=255), dict(rows=65)])
def test_matrices_that_do_not_belong_together(kw):
    for name in ("x", "wg", "wu"):
        if name == "x" and "rows" in kw:
            continue
        assert gated(**{name: mx(**kw)}) == B.PVT_EINVAL and grad(**{name: mx(**kw)}) == B.PVT_EINVAL
    assert grad_input(wu=mx(**kw)) == B.PVT_EINVAL


@pytest.mark.parametrize("act", [-1, 3])
def test_activations(act):
    assert gated(act=act) == B.PVT_EINVAL and grad(act=act) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(h=None), dict(h=0x8002), dict(dtype=3), dict(ld=63), dict(status=0x5002), dict(hq=mx(rows=4, cols=64)),
                                dict(hq=mx(rows=5, cols=65)), dict(hq=mx(rows=5, cols=64, format=B.PVT_MX_E4M3_16))])
def test_results_are_checked(kw):
    assert gated(**kw) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(dh=None), dict(dh=0x8002), dict(dtype=3), dict(ld=63), dict(dgate=None), dict(dgate=0x9008), dict(dup=None),
                                dict(dup=0xa002), dict(ldd=60), dict(ldd=56), dict(ldd=1 << 39), dict(dup=0x9000), dict(status=0x5001),
                                dict(dgate=0x8000), dict(dup=0x8000, dtype=B.PVT_BF16, ld=72)])
def test_gradients_are_checked(kw):
    assert grad(**kw) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(dgate=None), dict(dup=None), dict(dgate=0x9008), dict(dup=0xa008), dict(ldd=60), dict(ldd=56), dict(tokens=0),
                                dict(tokens=-1), dict(dx=None), dict(dx=0xb001), dict(dtype=3), dict(ld=255), dict(status=0x5003)])
def test_input_gradients_are_checked(kw):
    assert grad_input(**kw) == B.PVT_EINVAL


def test_one_sum_has_one_factor():
    fine = dict(format=B.PVT_MX_E4M3_16)
    assert grad_input(wg=mx(**fine, tensor_scale=0x3000), wu=mx(**fine, tensor_scale=0x3004)) == B.PVT_EINVAL
    assert grad_input(wg=mx(**fine), wu=mx(**fine, tensor_scale=0x3004)) == B.PVT_EINVAL
