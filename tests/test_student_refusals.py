"""The calls on the pass that g comes from reject bad arguments before anything is enqueued (no GPU: a call that launched
anything would say PVT_ECUDA)."""
import ctypes
import math

import pytest
import torch

import student_reference as ref
from paper_2405_14852_b200 import binding as B


def mx(**kw):
    base = dict(rows=64, cols=256, format=B.PVT_MX_E8M0_32, reserved_=0, ld=128, codes=0x1000, scales=0x2000, tensor_scale=None)
    base.update(kw)
    return B.pvt_mx(**base)


BAD_MX = [dict(rows=0), dict(rows=-1), dict(cols=0), dict(format=2), dict(format=-1), dict(codes=None), dict(codes=0x1008),
          dict(scales=None), dict(scales=0x2004), dict(ld=120), dict(ld=136), dict(ld=112), dict(ld=1 << 41),
          dict(tensor_scale=0x3000), dict(format=B.PVT_MX_E4M3_16, tensor_scale=0x3002), dict(rows=2 ** 31 - 1, cols=2 ** 31 - 1)]


@pytest.mark.parametrize("kw", BAD_MX)
def test_matrices_are_checked(kw):
    lib, m, good = B.lib(), mx(**kw), mx()
    before = B.pvt_launch_count()
    r = ctypes.byref
    assert lib.pvt_mx_quantize(r(m), 0x4000, B.PVT_F32, 1 << 33, None) == B.PVT_EINVAL
    assert lib.pvt_mx_dequant(r(m), 0x4000, B.PVT_F32, 1 << 33, None) == B.PVT_EINVAL
    assert lib.pvt_mx_product(r(m), r(good), 0x4000, B.PVT_F32, 1 << 33, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_product(r(good), r(m), 0x4000, B.PVT_F32, 1 << 33, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_grad_input(0x4000, 1 << 33, 4, r(m), 0x5000, B.PVT_F32, 1 << 33, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_grad_weight(0x4000, 1 << 33, 4, r(m), 0x5000, 1 << 33, 0, None, None) == B.PVT_EINVAL
    assert B.pvt_launch_count() == before


def test_null_matrices():
    lib = B.lib()
    assert lib.pvt_mx_quantize(None, 0x4000, B.PVT_F32, 256, None) == B.PVT_EINVAL
    assert lib.pvt_mx_product(None, ctypes.byref(mx()), 0x4000, B.PVT_F32, 64, None, None) == B.PVT_EINVAL


@pytest.mark.parametrize("ptr,dtype,ld", [(None, B.PVT_F32, 256), (0x4002, B.PVT_F32, 256), (0x4001, B.PVT_F16, 256),
                                          (0x4000, 3, 256), (0x4000, -1, 256), (0x4000, B.PVT_F32, 255), (0x4000, B.PVT_F32, 1 << 41)])
def test_float_matrices_are_checked(ptr, dtype, ld):
    lib, r = B.lib(), ctypes.byref
    m, x = mx(), mx(rows=3)
    assert lib.pvt_mx_quantize(r(m), ptr, dtype, ld, None) == B.PVT_EINVAL
    assert lib.pvt_mx_dequant(r(m), ptr, dtype, ld, None) == B.PVT_EINVAL
    wide = mx(rows=256)
    assert lib.pvt_mx_product(r(x), r(wide), ptr, dtype, ld, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_grad_input(0x8000, 64, 3, r(m), ptr, dtype, ld, None, None) == B.PVT_EINVAL


def test_products_of_unlike_matrices():
    lib, r = B.lib(), ctypes.byref
    assert lib.pvt_mx_product(r(mx()), r(mx(format=B.PVT_MX_E4M3_16)), 0x4000, B.PVT_F32, 64, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_product(r(mx()), r(mx(cols=255)), 0x4000, B.PVT_F32, 64, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_product(r(mx()), r(mx()), 0x4000, B.PVT_F32, 64, 0x5002, None) == B.PVT_EINVAL


@pytest.mark.parametrize("dy,ld,n", [(None, 64, 64), (0x4008, 64, 64), (0x4000, 60, 60), (0x4000, 56, 64), (0x4000, 64, 0),
                                     (0x4000, 64, -3), (0x4000, 1 << 39, 64)])
def test_gradients_are_checked(dy, ld, n):
    lib, r = B.lib(), ctypes.byref
    assert lib.pvt_mx_grad_weight(dy, ld, n, r(mx()), 0x5000, 256, 0, None, None) == B.PVT_EINVAL
    if n > 0:
        assert lib.pvt_mx_grad_input(dy, ld, 5, r(mx(rows=n)), 0x5000, B.PVT_F32, 256, None, None) == B.PVT_EINVAL
    assert lib.pvt_mx_grad_input(0x4000, 64, 0, r(mx()), 0x5000, B.PVT_F32, 256, None, None) == B.PVT_EINVAL


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 33), (128, 256), (129, 257), (1000, 5119), (28672, 8192)])
@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
def test_scale_bytes(rows, cols, fmt):
    assert B.pvt_mx_scale_bytes(rows, cols, fmt) == ref.scale_bytes(rows, cols, fmt)
    at = ref.scale_index(rows, min(cols, 600), fmt) if cols <= 600 else None
    if at is not None:
        assert at.max() < B.pvt_mx_scale_bytes(rows, cols, fmt) and at.unique().numel() == at.numel()


@pytest.mark.parametrize("args", [(0, 1, 0), (1, 0, 0), (1, 1, 2), (-1, 5, 1), (2 ** 31 - 1, 2 ** 31 - 1, 0)])
def test_scale_bytes_of_no_matrix(args):
    with pytest.raises(B.PvtError):
        B.pvt_mx_scale_bytes(*args)


def distill(**kw):
    base = dict(rows=3, vocab=100, k=5, logits=0x1000, ld=100, dtype=B.PVT_F32, temperature=1.0, top_idx=0x2000, top_logit=0x3000,
                teacher_lse=None, weight=None)
    base.update(kw)
    return B.pvt_distill(**base)


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=2 ** 31), dict(vocab=0), dict(vocab=2 ** 20 + 1), dict(k=0), dict(k=1025),
                                dict(logits=None), dict(logits=0x1002), dict(ld=99), dict(dtype=3), dict(temperature=0.0),
                                dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf),
                                dict(temperature=1e-39), dict(top_idx=None), dict(top_idx=0x2002), dict(top_logit=None),
                                dict(top_logit=0x3001), dict(teacher_lse=0x4002), dict(weight=0x4003)])
def test_distillations_are_checked(kw):
    lib, d = B.lib(), distill(**kw)
    before = B.pvt_launch_count()
    assert lib.pvt_distill_loss(ctypes.byref(d), 0x5000, None, None, None, 0, 0, None, None) == B.PVT_EINVAL
    assert lib.pvt_distill_grad(ctypes.byref(d), 0x5000, None, 0x6000, B.PVT_F32, 1 << 21, None, None) == B.PVT_EINVAL
    assert B.pvt_launch_count() == before


def test_outputs_of_distillations_are_checked():
    lib, d = B.lib(), ctypes.byref(distill())
    loss = lib.pvt_distill_loss
    assert loss(None, 0x5000, None, None, None, 0, 0, None, None) == B.PVT_EINVAL
    assert loss(d, None, None, None, None, 0, 0, None, None) == B.PVT_EINVAL
    assert loss(d, 0x5001, None, None, None, 0, 0, None, None) == B.PVT_EINVAL
    assert loss(d, 0x5000, 0x6001, None, None, 0, 0, None, None) == B.PVT_EINVAL
    assert loss(d, 0x5000, None, 0x6002, None, 0, 0, None, None) == B.PVT_EINVAL
    assert loss(d, 0x5000, None, None, 0x6000, 7, 100, None, None) == B.PVT_EINVAL
    assert loss(d, 0x5000, None, None, 0x6000, B.PVT_F32, 99, None, None) == B.PVT_EINVAL
    assert loss(d, 0x5000, None, None, 0x1000, B.PVT_BF16, 100, None, None) == B.PVT_EINVAL  # in place, another type
    assert loss(d, 0x5000, None, None, 0x1000, B.PVT_F32, 104, None, None) == B.PVT_EINVAL   # in place, other rows
    assert loss(d, 0x5000, None, None, None, 0, 0, 0x7002, None) == B.PVT_EINVAL
    grad = lib.pvt_distill_grad
    assert grad(d, None, None, 0x6000, B.PVT_F32, 100, None, None) == B.PVT_EINVAL
    assert grad(d, 0x5000, None, None, B.PVT_F32, 100, None, None) == B.PVT_EINVAL
    assert grad(d, 0x5000, None, 0x1000, B.PVT_F16, 100, None, None) == B.PVT_EINVAL


@pytest.mark.parametrize("kw", [dict(logits=None), dict(logits=0x1001), dict(dtype=9), dict(ld=99), dict(rows=0), dict(vocab=0),
                                dict(vocab=2 ** 20 + 1), dict(k=0), dict(k=101), dict(k=1025), dict(temperature=0.0),
                                dict(temperature=math.nan), dict(idx=None), dict(idx=0x2002), dict(val=None), dict(val=0x3002),
                                dict(lse=0x4001)])
def test_lists_are_checked(kw):
    a = dict(logits=0x1000, dtype=B.PVT_F16, ld=100, rows=4, vocab=100, k=10, temperature=1.0, idx=0x2000, val=0x3000, lse=0x4000)
    a.update(kw)
    rc = B.lib().pvt_distill_top(a["logits"], a["dtype"], a["ld"], a["rows"], a["vocab"], a["k"], a["temperature"], a["idx"],
                                 a["val"], a["lse"], None)
    assert rc == B.PVT_EINVAL


def test_the_binding_refuses_tensors_that_do_not_fit():
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(1024, dtype=torch.uint8)
    for bad in (lambda: B.make_mx(codes, scales, 4, 64, B.PVT_MX_E8M0_32),                # not on a GPU
                lambda: B.make_mx(codes, scales, 5, 64, B.PVT_MX_E8M0_32),
                lambda: B.make_mx(codes[:, :24], scales, 4, 48, B.PVT_MX_E8M0_32),
                lambda: B.make_mx(codes, scales, 4, 65, B.PVT_MX_E8M0_32),                # a row of 33 bytes
                lambda: B.make_mx(codes, scales, 4, 64, 5),
                lambda: B.make_mx(codes, scales[:1000], 4, 64, B.PVT_MX_E8M0_32),
                lambda: B.make_mx(codes, scales, 0, 64, B.PVT_MX_E8M0_32),
                lambda: B.make_mx(codes.int(), scales, 4, 64, B.PVT_MX_E8M0_32),
                lambda: B.make_mx(codes, scales, 4, 64, B.PVT_MX_E8M0_32, tensor_scale=torch.ones(1)),
                lambda: B.make_distill(torch.zeros(2, 9), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)),
                lambda: B.make_distill(torch.zeros(2, 9), torch.zeros(2, 3), torch.zeros(2, 3)),
                lambda: B.make_distill(torch.zeros(2, 9).double(), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)),
                lambda: B.make_distill(torch.zeros(9, 2).T, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)),
                lambda: B.pvt_distill_top(torch.zeros(2, 9), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3))):
        with pytest.raises(ValueError):
            bad()


def test_the_reference_quantiser_takes_the_nearest_element_and_scale():
    """The checker's own codes against a search of all elements and all scales (float64)."""
    x = torch.randn(6, 64, dtype=torch.float64) * torch.exp2(torch.randint(-6, 6, (6, 1)).double())
    for fmt, ts in ((ref.E8M0, None), (ref.E4M3, None), (ref.E4M3, 0.0041)):
        codes, scales = ref.quantize(x, fmt, ts)
        b = ref.BLOCK[fmt]
        table = ref.scale_values(fmt)
        for r in range(6):
            for n in range(64 // b):
                block = x[r, n * b:(n + 1) * b]
                s = table[scales[r, n]] * (1.0 if ts is None else ts)
                err = (ref.element_values()[:, None] * s - block[None]).abs()
                got = ref.element_values()[codes[r, n * b:(n + 1) * b]] * s
                assert torch.allclose((got - block).abs(), err.min(dim=0).values, rtol=0, atol=1e-15)
                if fmt == ref.E4M3:
                    want = block.abs().max() / (6 * (1.0 if ts is None else ts))
                    finite = table[:127]
                    assert abs(finite[scales[r, n]] - want) <= (finite - want).abs().min() + 1e-15
                else:
                    top = block.abs().max()
                    assert table[scales[r, n]] * 4 <= top < table[scales[r, n]] * 8


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
def test_scale_bytes_of_the_longest_rows(fmt):
    cols = 2 ** 31 - 1
    assert B.pvt_mx_scale_bytes(1, cols, fmt) == ref.scale_bytes(1, cols, fmt)


def test_temperatures_whose_reciprocal_is_beyond_the_kernels_numbers():
    """log2(e) / temperature has to be a finite binary32: at 3.4e-39 the reciprocal is, 1.44 times it is not."""
    lib, d = B.lib(), distill(temperature=3.4e-39)
    assert lib.pvt_distill_loss(ctypes.byref(d), 0x5000, None, None, None, 0, 0, None, None) == B.PVT_EINVAL
    assert lib.pvt_distill_top(0x1000, B.PVT_F16, 100, 4, 100, 10, 3.4e-39, 0x2000, 0x3000, None, None) == B.PVT_EINVAL
