"""The norm at batches, where a team of threads has two rows at a time and goes round its ring many times; rows that are no numbers under
either kind."""
import math

import pytest
import torch

import block_reference as ref
import student_reference as mx
from paper_2405_14852_b200 import binding as B
from test_gpu_norm import TYPES, check_held, close, rows, weights

pytestmark = pytest.mark.gpu

KINDS = [B.PVT_NORM_LAYER, B.PVT_NORM_RMS]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [64, 200, 1500, 9000])
def test_rows_with_nan_infinity_or_squares_beyond_binary32(kind, cols):
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(40, cols, device="cuda", generator=gen)
    w, b = weights(gen, cols, torch.float32)
    bad = x.clone()
    bad[3, cols // 2], bad[7, 0], bad[39, cols - 1], bad[20] = math.nan, math.inf, -math.inf, bad[20] * 1e30
    out, want = torch.empty_like(x), torch.empty_like(x)
    stats = torch.empty(40, 2, device="cuda")
    B.pvt_norm_apply(B.make_norm(x, w, b, kind=kind), y=want)
    fine = torch.ones(40, dtype=torch.bool, device="cuda")
    fine[[3, 7, 39, 20]] = False
    for fmt in (B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16):
        m = B.new_mx(40, cols, fmt)
        B.pvt_norm_apply(B.make_norm(bad, w, b, kind=kind), y=out, quantized=m, stats=stats)
        assert torch.equal(out[fine], want[fine]) and torch.isnan(out[3]).all()
        assert stats[20, 1] == 0 and torch.equal(out[20], b)
        check_held(m, out, fmt)
        if kind == B.PVT_NORM_LAYER:
            assert torch.isnan(out[[7, 39]]).all()
        else:
            assert (stats[[7, 39], 1] == 0).all()
            for row, col in ((7, 0), (39, cols - 1)):
                rest = torch.arange(cols, device="cuda") != col
                assert torch.isnan(out[row, col]) and torch.equal(out[row, rest], b[rest])


def together(rows, cols, floats_without_mean=False):
    """Whether aligned rows are taken two at a time on 148 SMs, by the rule of the launch, of 16-bit types."""
    spans = -(-cols // 256)
    teams = 256 // (8 if cols <= 64 else 16 if cols <= 128 else 32) if spans == 1 else 1
    threads = 256 if spans == 1 else 32 * (spans if spans <= 4 else -(-spans // 2))
    at_once = 148 * (512 // threads) * teams
    return rows > 2 * at_once and not (floats_without_mean and rows > 4 * at_once)


# two rows at a time with one block to a row, teams of 8, 16 and 32 lanes among them, many rounds of the ring, a last round that not all
# teams have; whole spans and others; and where floats without the mean go back to one row at a time
BATCHES = [(700, 4096), (1500, 4096), (400, 8192), (1301, 8192), (2100, 2048), (5003, 2048), (20011, 64), (40003, 40), (15013, 128),
           (30011, 256), (5009, 512), (9001, 520), (1303, 4008), (3001, 1000), (7013, 1024)]


@pytest.mark.parametrize("case,shape", list(enumerate(BATCHES)))
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("with_residual", [False, True])
def test_batches_of_rows(case, shape, kind, with_residual):
    """types change from case to case"""
    gen = torch.Generator("cuda").manual_seed(10 * case + kind)
    n = case + kind + 2 * with_residual
    dtype, out, w_type, pad = TYPES[n % 3], TYPES[(n // 2) % 3], TYPES[(n + 1) % 3], 8 * (n % 2)
    x = rows(gen, shape, dtype, pad, offset=2.0 if n % 5 == 0 else 0.1)
    residual = rows(gen, shape, dtype, pad) if with_residual else None
    w, b = weights(gen, shape[1], w_type)
    y, stats = torch.full((shape[0], shape[1] + pad), 7.0, dtype=out, device="cuda"), torch.full((shape[0] + 1, 2), 7.0, device="cuda")
    total = torch.full((shape[0], shape[1] + pad), 7.0, dtype=dtype, device="cuda")
    B.pvt_norm_apply(B.make_norm(x, w, b, kind=kind, residual=residual), y=y[:, :shape[1]], total=total[:, :shape[1]], stats=stats[:-1])
    r = (x.float() + residual.float()).to(dtype) if with_residual else x
    assert torch.equal(total[:, :shape[1]], r)
    assert (y[:, shape[1]:] == 7).all() and (total[:, shape[1]:] == 7).all() and (stats[-1] == 7).all()
    want, mean, rstd = ref.norm(r, kind, 1e-5, w, b)
    d_y, d_mean, d_rstd = ref.norm_bounds(r, kind, 1e-5, w, b)
    close(stats[:-1, :1], mean, d_mean)
    close(stats[:-1, 1:], rstd, d_rstd)
    close(y[:, :shape[1]], want, d_y, out)


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case,shape", list(enumerate([(700, 4096), (400, 8192), (2100, 2048), (5003, 2048), (1303, 4008), (3001, 1000),
                                                       (6007, 200), (12011, 256)])))
def test_batches_of_rows_into_four_bits(fmt, kind, case, shape):
    gen = torch.Generator("cuda").manual_seed(50 + case)
    dtype = TYPES[(case + kind) % 3]
    x, residual = rows(gen, shape, dtype, 8), rows(gen, shape, dtype, 8) if case % 2 else None
    w, b = weights(gen, shape[1], torch.float32)
    ts = torch.tensor([0.002], device="cuda") if fmt == B.PVT_MX_E4M3_16 and kind else None
    m = B.new_mx(*shape, fmt, ts)
    m.codes.fill_(0xa5), m.scales.fill_(0xa5)
    y = torch.empty(shape, device="cuda")
    n = B.make_norm(x, w, b, kind=kind, residual=residual)
    B.pvt_norm_apply(n, y=y, quantized=m)
    r = x if residual is None else (x.float() + residual.float()).to(dtype)
    close(y, ref.norm(r, kind, 1e-5, w, b)[0], ref.norm_bounds(r, kind, 1e-5, w, b)[0])
    check_held(m, y, fmt, ts)
    keep = m.codes.clone(), m.scales.clone()
    m.codes.fill_(0xa5), m.scales.fill_(0xa5)
    B.pvt_norm_apply(n, quantized=m)  # and by itself, as a student's pass has it
    used = (shape[1] + 1) // 2
    assert torch.equal(m.codes[:, :used], keep[0][:, :used]) and torch.equal(m.scales, keep[1])


@pytest.mark.parametrize("case,shape", list(enumerate([(3001, 1000), (1200, 8192), (9001, 96), (20011, 64), (1500, 4096), (5003, 2048), (700, 16384),
                                                       (2003, 4001), (6007, 255)])))
@pytest.mark.parametrize("kind", KINDS)
def test_gradients_of_batches(case, shape, kind):
    """Many rounds of the ring; rows of no alignment last."""
    gen = torch.Generator("cuda").manual_seed(500 + case)
    n = case + kind
    dtype, g_type = TYPES[n % 3], TYPES[(n + 1) % 3]
    x = rows(gen, shape, dtype, 0, offset=0.1)
    _, mean, rstd = ref.norm(x, kind, 1e-5)
    stats = torch.cat((mean, rstd), dim=1).float()
    dy, res = rows(gen, shape, g_type), rows(gen, shape, g_type) if n % 2 else None
    w = weights(gen, shape[1], torch.float32)[0]
    dx = torch.empty(shape, dtype=g_type, device="cuda")
    dw, db = torch.empty(shape[1], device="cuda"), torch.empty(shape[1], dtype=torch.float64, device="cuda")
    d = B.make_norm(x, w, kind=kind)
    ws = B.new_norm_workspace(d).fill_(0xff)
    B.pvt_norm_grad(d, stats, dy, dx, dresidual=res, dweight=dw, workspace=ws)
    want, bounds = ref.norm_grad(x, stats, dy, kind, w, res), ref.norm_grad_bounds(x, stats, dy, kind, w, res)
    close(dx, want[0], bounds[0], g_type)
    close(dw, want[1], bounds[1], torch.float32)
    B.pvt_norm_grad(d, stats, dy, dx, dresidual=res, dbias=db, workspace=ws)
    close(db, want[2], bounds[2], torch.float32)


def test_the_cases_are_the_ones_they_are_for():
    two = [s for s in BATCHES if together(*s)]
    assert len(two) >= 12 and {64, 40, 128, 256, 512, 2048, 4096, 8192} <= {c for _, c in two}
    assert any(together(*s, floats_without_mean=True) for s in BATCHES) and any(together(*s) and not together(*s, floats_without_mean=True) for s in BATCHES)
