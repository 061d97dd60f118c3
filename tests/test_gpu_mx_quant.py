"""Quantisation to 4-bit block floating point and back, against tables and comparisons in float64.

Codes and scales are whole numbers: every one of them has to be equal, at borders between two elements or two scales too."""
import math

import pytest
import torch

import student_reference as ref
from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

FORMATS = [(B.PVT_MX_E8M0_32, None), (B.PVT_MX_E4M3_16, None), (B.PVT_MX_E4M3_16, 0.00037)]


def quantized(x, fmt, ts=None):
    rows, cols = x.shape
    scale = None if ts is None else torch.tensor([ts], dtype=torch.float32, device="cuda")
    m = B.new_mx(rows, cols, fmt, tensor_scale=scale)
    m.codes.fill_(0xa5)
    m.scales.fill_(0xa5)
    B.pvt_mx_quantize(m, x)
    return m


def check(x, fmt, ts=None):
    rows, cols = x.shape
    m = quantized(x, fmt, ts)
    f32 = None if ts is None else m.tensor_scale.item()
    codes, scales = ref.quantize(x, fmt, f32)
    want_codes, want_scales = ref.pack(codes, scales, fmt, fill=0xa5)
    got_codes, got_scales = ref.unpack(m.codes, m.scales, rows, cols, fmt)
    assert torch.equal(got_scales, scales)
    assert torch.equal(got_codes, codes)
    assert torch.equal(m.codes, want_codes)    # an odd row's last half byte is 0, what lies behind it is as it was
    assert torch.equal(m.scales, want_scales)  # scales of rows and blocks that do not exist are 0
    out = torch.empty(rows, cols, device="cuda")
    B.pvt_mx_dequant(m, out)
    want = ref.values(codes, scales, fmt, f32).float()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(out.nan_to_num(), want.nan_to_num())
    return m, want


@pytest.mark.parametrize("fmt,ts", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 33), (2, 255), (1, 4096), (129, 256), (130, 1001), (257, 2048)])
def test_codes_scales_and_values(rows, cols, dtype, fmt, ts):
    gen = torch.Generator(device="cuda").manual_seed(rows * 10007 + cols)
    x = (torch.randn(rows, cols, device="cuda", generator=gen) * 0.02 *
         torch.exp(2 * torch.randn(rows, 1, device="cuda", generator=gen))).to(dtype)
    check(x, fmt, ts)


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (8, 8), (1, 15)])
def test_rows_of_any_alignment(fmt, offset, pad):
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.randn(37, offset + 517 + pad, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(dtype)
        check(wide[:, offset:offset + 517], fmt)


@pytest.mark.parametrize("fmt,ts", FORMATS)
def test_borders(fmt, ts):
    """Elements on every border between two codes and one step of binary32 to either side of it, under many scales."""
    step = 1.0 if ts is None else float(torch.tensor(ts, dtype=torch.float32))
    borders = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]
    rows = []
    for s in ([2.0 ** e for e in range(-20, 20, 3)] if fmt == B.PVT_MX_E8M0_32
              else [ref.E4M3_VALUES[i] for i in range(1, 127, 5)]):
        for shift in (-1, 0, 1):
            row = torch.tensor([b * s * step * sign for b in borders for sign in (1, -1)], dtype=torch.float64).float()
            row = (row.view(torch.int32) + shift).view(torch.float32)
            row[-1] = -6.0 * s * step  # sets the scale
            rows.append(torch.cat([row, row]))
    check(torch.stack(rows).cuda(), fmt, ts)


@pytest.mark.parametrize("ts", [None, 0.00037, 1.7e-30, 3.1e30])
def test_borders_of_the_scale(ts):
    """The largest element on every midpoint between two e4m3 scales and next to it; scales that vanish or saturate."""
    step = 1.0 if ts is None else float(torch.tensor(ts, dtype=torch.float32))
    values = ref.E4M3_VALUES
    points = [0.5 * (a + b) * 6 * step for a, b in zip(values[:-1], values[1:])] + [448 * 6 * step, 2000 * 6 * step]
    rows = []
    for shift in (-1, 0, 1):
        for a in points:
            row = torch.linspace(-1, 1, 16, dtype=torch.float64) * a
            row = row.float()
            row[3] = (torch.tensor([a]).float().view(torch.int32) + shift).view(torch.float32)
            row = torch.where(row.abs() > row[3], row[3], row)
            rows.append(row)
    check(torch.stack(rows).cuda(), B.PVT_MX_E4M3_16, ts)


@pytest.mark.parametrize("fmt,ts", FORMATS)
def test_numbers_at_the_ends_of_the_range(fmt, ts):
    tiny, big = 2.0 ** -149, 3.4e38
    x = torch.zeros(8, 64)
    x[0, :] = tiny
    x[1, 5] = -big
    x[1, 20] = 1.0
    x[2, 40] = 2.0 ** -126
    x[3, :] = -0.0
    x[4, 33] = 2.0 ** -127 * 1.5
    x[5, 0:32] = torch.linspace(-big, big, 32)
    x[6, 1] = 2.0 ** -125
    check(x.cuda(), fmt, ts)


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_block_that_is_not_finite_is_nan_and_its_neighbours_are_not(fmt, bad):
    x = torch.randn(3, 200, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    x[1, 70] = bad
    x[2, 199] = bad
    _, want = check(x, fmt)
    assert torch.isnan(want).sum().item() == (32 + 8 if fmt == B.PVT_MX_E8M0_32 else 16 + 8)


@pytest.mark.parametrize("ts", [0.0, -1.0, math.nan, math.inf])
def test_a_tensor_scale_that_is_no_scale_gives_nan(ts):
    x = torch.randn(2, 40, device="cuda")
    _, want = check(x, B.PVT_MX_E4M3_16, ts)
    assert torch.isnan(want).all()


@pytest.mark.parametrize("fmt,ts", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_values_in_16_bits_are_rounded_once(fmt, ts, dtype):
    x = torch.randn(65, 301, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    m = quantized(x, fmt, ts)
    wide = torch.full((65, 320), 7.0, dtype=dtype, device="cuda")
    B.pvt_mx_dequant(m, wide[:, 9:310])
    codes, scales = ref.unpack(m.codes, m.scales, 65, 301, fmt)
    want = ref.values(codes, scales, fmt, None if ts is None else m.tensor_scale.item()).float().to(dtype)
    assert torch.equal(wide[:, 9:310], want)
    assert (wide[:, :9] == 7).all() and (wide[:, 310:] == 7).all()


def test_quantising_values_again_changes_nothing():
    x = torch.randn(40, 640, device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    a = quantized(x, B.PVT_MX_E8M0_32)
    v = torch.empty(40, 640, device="cuda")
    B.pvt_mx_dequant(a, v)
    w = torch.empty(40, 640, device="cuda")
    B.pvt_mx_dequant(quantized(v, B.PVT_MX_E8M0_32), w)
    assert torch.equal(v, w)


def test_codes_in_wider_rows_leave_what_lies_beside_them():
    x = torch.randn(5, 75, device="cuda")
    wide = torch.full((5, 96), 0x5a, dtype=torch.uint8, device="cuda")
    scales = torch.empty(B.pvt_mx_scale_bytes(5, 75, B.PVT_MX_E8M0_32), dtype=torch.uint8, device="cuda")
    m = B.make_mx(wide[:, 16:64], scales, 5, 75, B.PVT_MX_E8M0_32)
    B.pvt_mx_quantize(m, x)
    codes, _ = ref.quantize(x, B.PVT_MX_E8M0_32)
    got, _ = ref.unpack(wide[:, 16:64], scales, 5, 75, B.PVT_MX_E8M0_32)
    assert torch.equal(got, codes)
    assert (wide[:, :16] == 0x5a).all() and (wide[:, 16 + 38:] == 0x5a).all()


@pytest.mark.parametrize("ts", [1.5e-45, 1e-40, 1.2e-38, 5.6e37, 6e37, 3.4e38])
def test_tensor_scales_at_the_ends_of_the_range(ts):
    """6 tensor_scale or its reciprocal is no normal number there."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    wide = torch.exp(torch.linspace(-100, 88, 70, device="cuda"))[:, None]
    check(torch.rand(70, 64, device="cuda", generator=gen) * wide, B.PVT_MX_E4M3_16, ts)
    check(torch.full((2, 48), 3.4e38, device="cuda"), B.PVT_MX_E4M3_16, ts)


def test_rows_further_apart_than_32_bits_count():
    """Elements and codes whose offsets pass 2^32 bytes."""
    rows, cols, apart = 3, 700, 2 ** 31 + 64
    codes = torch.empty(2 * apart + 4096, dtype=torch.uint8, device="cuda").as_strided((rows, 352), (apart, 1))
    x = torch.empty(2 * apart + 4096, dtype=torch.bfloat16, device="cuda").as_strided((rows, cols), (apart, 1))
    x.copy_(torch.randn(rows, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(7)))
    for fmt in (B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16):
        scales = torch.empty(B.pvt_mx_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda")
        m = B.make_mx(codes, scales, rows, cols, fmt)
        B.pvt_mx_quantize(m, x)
        want, want_scales = ref.quantize(x, fmt)
        got, got_scales = ref.unpack(codes, scales, rows, cols, fmt)
        assert torch.equal(got, want) and torch.equal(got_scales, want_scales)
        v = ref.values(want, want_scales, fmt)
        near = B.new_mx(rows, cols, fmt)
        B.pvt_mx_quantize(near, torch.ones(rows, cols, device="cuda"))
        y = torch.empty(rows, rows, device="cuda")
        B.pvt_mx_product(m, near, y)
        ones = ref.values(*ref.unpack(near.codes, near.scales, rows, cols, fmt), fmt)
        assert ((y.double() - v @ ones.T).abs() <= (cols + 4) * 2.0 ** -23 * (v.abs() @ ones.T)).all()
        far = torch.empty(2 * apart + 4096, dtype=torch.bfloat16, device="cuda").as_strided((rows, cols), (apart, 1))
        B.pvt_mx_dequant(m, far)
        assert torch.equal(far, v.bfloat16())
        dy = torch.eye(rows, 8, dtype=torch.bfloat16, device="cuda")[:, :rows]
        B.pvt_mx_grad_input(dy, m, far)
        assert torch.equal(far, v.bfloat16())
        del far


@pytest.mark.parametrize("fmt,ts", FORMATS)
@pytest.mark.parametrize("rows,cols", [(5, 8), (300, 21), (257, 32), (129, 33), (1000, 64), (2, 100), (515, 127), (1025, 128), (20000, 31)])
def test_rows_of_few_columns(rows, cols, fmt, ts):
    """Several rows share a warp: rows of any distance, and values that lie beside others."""
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    for dtype, pad in ((torch.float32, 0), (torch.bfloat16, 3), (torch.float16, 8)):
        wide = torch.full((rows, cols + pad), math.nan, device="cuda", dtype=dtype)
        wide[:, :cols] = (torch.randn(rows, cols, device="cuda", generator=gen) *
                          torch.exp(3 * torch.randn(rows, 1, device="cuda", generator=gen))).to(dtype)
        if rows > 2:
            wide[1, cols // 2] = math.inf
        m, want = check(wide[:, :cols], fmt, ts)
        out = torch.full((rows, cols + 5), 7.0, device="cuda", dtype=dtype)
        B.pvt_mx_dequant(m, out[:, 2:cols + 2])
        assert torch.equal(out[:, 2:cols + 2].isnan(), want.isnan())
        assert torch.equal(out[:, 2:cols + 2].nan_to_num(), want.to(dtype).nan_to_num())
        assert (out[:, :2] == 7).all() and (out[:, cols + 2:] == 7).all()
