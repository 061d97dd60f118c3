"""The norm ahead of a layer and its gradients against the formulas in float64: every width class of the kernels, types, rows of no
alignment, 4-bit results, results in the place of operands, gradients against differences, streams, graphs, refusals by the binding."""
import math

import pytest
import torch

import block_reference as ref
import student_reference as mx
from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
# widths of one lane team (8, 16 and 32 lanes), of a warp, of a block by one to eight spans to a warp, of a cluster of two and four
SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (1001, 64), (9, 65), (700, 128), (33, 129), (40, 256), (7, 257), (300, 512), (5, 1000),
          (149, 1024), (2, 2047), (600, 2048), (5, 4096), (300, 4100), (3, 5001), (160, 8192), (5, 8193), (150, 16384), (4, 20001),
          (151, 20480), (2, 32768), (1, 32767)]


def rows(gen, shape, dtype, pad=0, std=1.0, offset=0.0):
    """A matrix cut out of a wider one that is NaN elsewhere."""
    wide = torch.full((shape[0], shape[1] + pad), math.nan, dtype=dtype, device="cuda")
    wide[:, :shape[1]] = std * torch.randn(shape, device="cuda", generator=gen) + offset
    return wide[:, :shape[1]]


def weights(gen, cols, dtype):
    return ((1 + 0.3 * torch.randn(cols, device="cuda", generator=gen)).to(dtype),
            (0.2 * torch.randn(cols, device="cuda", generator=gen)).to(dtype))


def close(got, want, bound, dtype=None):
    slack = bound + (ref.rounding(want.abs() + bound, dtype) if dtype is not None else 0.0)
    assert got.shape == want.shape
    off = (got.double() - want).abs()
    assert (off <= slack).all(), f"off by up to {(off / slack).max().item():.3g} of what is allowed"


def check_held(m, values, fmt, ts=None):
    """codes and scales are those of quantising `values`"""
    codes, scales = mx.quantize(values, fmt, None if ts is None else ts.item())
    got_codes, got_scales = mx.unpack(m.codes, m.scales, m.rows, m.cols, fmt)
    assert torch.equal(got_scales, scales) and torch.equal(got_codes, codes)
    held, packed = mx.pack(codes, scales, fmt)
    assert torch.equal(m.scales, packed)  # those of rows and blocks that do not exist are 0


@pytest.mark.parametrize("case,shape", list(enumerate(SHAPES)))
@pytest.mark.parametrize("kind", [B.PVT_NORM_LAYER, B.PVT_NORM_RMS])
def test_norm(case, shape, kind):
    """types, residual, bias and the distance of rows change from case to case"""
    gen = torch.Generator("cuda").manual_seed(100 * case + kind)
    n = case + kind
    dtype, out, w_type, pad = TYPES[n % 3], TYPES[(n // 3) % 3], TYPES[(n // 2) % 3], [0, 0, 8, 1][n % 4]
    x = rows(gen, shape, dtype, pad, offset=3.0 if n % 5 == 0 else 0.1)
    residual = rows(gen, shape, dtype, pad) if n % 2 else None
    w, b = weights(gen, shape[1], w_type)
    w, b = (w, b) if kind == B.PVT_NORM_LAYER else (w, None) if n % 3 else (None, None)
    y = torch.full((shape[0], shape[1] + pad), 7.0, dtype=out, device="cuda")
    total = torch.full((shape[0], shape[1] + pad), 7.0, dtype=dtype, device="cuda")
    stats = torch.full((shape[0] + 1, 2), 7.0, device="cuda")
    B.pvt_norm_apply(B.make_norm(x, w, b, kind=kind, eps=1e-5, residual=residual), y=y[:, :shape[1]], total=total[:, :shape[1]],
                     stats=stats[:-1])
    r = x if residual is None else (x.float() + residual.float()).to(dtype)
    assert torch.equal(total[:, :shape[1]], r)
    assert (y[:, shape[1]:] == 7).all() and (total[:, shape[1]:] == 7).all() and (stats[-1] == 7).all()
    want, mean, rstd = ref.norm(r, kind, 1e-5, w, b)
    d_y, d_mean, d_rstd = ref.norm_bounds(r, kind, 1e-5, w, b)
    close(stats[:-1, :1], mean, d_mean)
    close(stats[:-1, 1:], rstd, d_rstd)
    close(y[:, :shape[1]], want, d_y, out)


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("case,shape", list(enumerate([(1, 1), (1, 40), (3, 100), (130, 255), (129, 256), (2, 300), (1, 2048), (200, 1030),
                                                  (5, 4096), (150, 5001), (3, 8192), (2, 16385), (1, 32768)])))
def test_norm_into_four_bits(fmt, case, shape):
    gen = torch.Generator("cuda").manual_seed(case)
    dtype, pad = TYPES[case % 3], [0, 1, 8][case % 3]
    x, residual = rows(gen, shape, dtype, pad), rows(gen, shape, dtype, pad) if case % 2 else None
    w, b = weights(gen, shape[1], TYPES[(case + 1) % 3])
    ts = torch.tensor([0.01], device="cuda") if fmt == B.PVT_MX_E4M3_16 and case % 4 else None
    pitch = -(-shape[1] // 32) * 16 + 16
    codes = torch.full((shape[0], pitch), 0xa5, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.pvt_mx_scale_bytes(*shape, fmt),), 0xa5, dtype=torch.uint8, device="cuda")
    m = B.make_mx(codes, scales, *shape, fmt, tensor_scale=ts)
    y = torch.empty(shape, device="cuda")
    n = B.make_norm(x, w, b, residual=residual)
    B.pvt_norm_apply(n, y=y, quantized=m)
    check_held(m, y, fmt, ts)
    assert (codes[:, (shape[1] + 1) // 2:] == 0xa5).all()
    keep = codes.clone(), scales.clone()
    codes.fill_(0xa5), scales.fill_(0xa5)
    B.pvt_norm_apply(n, quantized=m)  # and by itself
    assert torch.equal(codes, keep[0]) and torch.equal(scales, keep[1])


@pytest.mark.parametrize("case,shape", list(enumerate(SHAPES)))
@pytest.mark.parametrize("kind", [B.PVT_NORM_LAYER, B.PVT_NORM_RMS])
def test_gradients(case, shape, kind):
    gen = torch.Generator("cuda").manual_seed(1000 + 100 * case + kind)
    n = case + 2 * kind
    dtype, g_type, w_type, pad = TYPES[n % 3], TYPES[(n // 3) % 3], TYPES[(n // 2) % 3], [0, 0, 8, 1][n % 4]
    x = rows(gen, shape, dtype, pad, offset=2.0 if n % 5 == 0 else 0.1)
    _, mean, rstd = ref.norm(x, kind, 1e-5)
    stats = torch.cat((mean, rstd), dim=1).float()
    dy = rows(gen, shape, g_type, pad)
    res = rows(gen, shape, g_type, pad) if n % 2 else None
    w = weights(gen, shape[1], w_type)[0] if n % 4 else None
    dx = torch.full((shape[0], shape[1] + pad), 7.0, dtype=g_type, device="cuda")
    dw_type = [torch.float32, torch.float64][case % 2]
    dw, db = torch.full((shape[1] + 1,), 7.0, dtype=dw_type, device="cuda"), torch.full((shape[1] + 1,), 7.0, dtype=dw_type, device="cuda")
    d = B.make_norm(x, w, kind=kind)
    ws = B.new_norm_workspace(d).fill_(0xff)
    B.pvt_norm_grad(d, stats, dy, dx[:, :shape[1]], dresidual=res, dweight=dw[:-1], dbias=db[:-1], workspace=ws)
    want = ref.norm_grad(x, stats, dy, kind, w, res)
    bounds = ref.norm_grad_bounds(x, stats, dy, kind, w, res)
    close(dx[:, :shape[1]], want[0], bounds[0], g_type)
    close(dw[:-1], want[1], bounds[1], F32)
    close(db[:-1], want[2], bounds[2], F32)
    assert (dx[:, shape[1]:] == 7).all() and dw[-1] == 7 and db[-1] == 7
    # the same again, added to; one of the two alone; neither
    keep = dx.clone(), dw.clone(), db.clone()
    B.pvt_norm_grad(d, stats, dy, dx[:, :shape[1]], dresidual=res, dweight=dw[:-1], dbias=db[:-1], accumulate=True, workspace=ws)
    assert torch.equal(dx, keep[0])
    close(dw[:-1], keep[1][:-1].double() + want[1], bounds[1], F32)
    close(db[:-1], keep[2][:-1].double() + want[2], bounds[2], F32)
    for which in ((dw, None), (None, db), (None, None)):
        dx.fill_(7.0), dw.fill_(7.0), db.fill_(7.0)
        B.pvt_norm_grad(d, stats, dy, dx[:, :shape[1]], dresidual=res, dweight=which[0] if which[0] is None else dw[:-1],
                        dbias=which[1] if which[1] is None else db[:-1], workspace=ws if any(t is not None for t in which) else None)
        assert torch.equal(dx, keep[0])
        assert torch.equal(dw, keep[1]) if which[0] is not None else (dw == 7).all()
        assert torch.equal(db, keep[2]) if which[1] is not None else (db == 7).all()


@pytest.mark.parametrize("kind", [B.PVT_NORM_LAYER, B.PVT_NORM_RMS])
def test_gradients_against_differences(kind):
    """The formula of the gradients is the derivative of the formula of the norm, and the kernel's is the formula's."""
    gen = torch.Generator("cuda").manual_seed(5)
    x, dy = (torch.randn(6, 37, dtype=torch.float64, device="cuda", generator=gen) for _ in range(2))
    w, b = (torch.randn(37, dtype=torch.float64, device="cuda", generator=gen) for _ in range(2))
    _, mean, rstd = ref.norm(x, kind, 1e-5)
    got = ref.norm_grad(x, torch.cat((mean, rstd), dim=1), dy, kind, w)

    def loss(x, w, b):
        return (ref.norm(x, kind, 1e-5, w, b)[0] * dy).sum()

    h = 1e-6
    for at, t in ((0, x), (1, w), (2, b)):
        flat, want = t.view(-1), got[at].reshape(-1)
        for i in range(0, flat.numel(), 5):
            keep = flat[i].item()
            flat[i] = keep + h
            up = loss(x, w, b)
            flat[i] = keep - h
            down = loss(x, w, b)
            flat[i] = keep
            assert abs((up - down).item() / (2 * h) - want[i].item()) <= 1e-6 * (1 + abs(want[i].item()))
    stats = torch.cat((mean, rstd), dim=1).float()
    dx, dw, db = torch.empty(6, 37, device="cuda"), torch.empty(37, device="cuda"), torch.empty(37, device="cuda")
    d = B.make_norm(x.float(), w.float(), kind=kind)
    B.pvt_norm_grad(d, stats, dy.float(), dx, dweight=dw, dbias=db, workspace=B.new_norm_workspace(d))
    for have, want in zip((dx, dw, db), got):
        assert (have.double() - want).abs().max() <= 1e-5 * want.abs().max()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,pad", [(200, 0), (1000, 3), (4096, 8), (20000, 0)])
def test_results_in_the_place_of_operands(dtype, cols, pad):
    gen = torch.Generator("cuda").manual_seed(cols)
    shape = (70, cols)
    x, res = rows(gen, shape, dtype, pad), rows(gen, shape, dtype, pad)
    w, b = weights(gen, cols, dtype)
    y, total, stats = torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(70, 2, device="cuda")
    B.pvt_norm_apply(B.make_norm(x, w, b, residual=res), y=y, total=total, stats=stats)
    x2, r2 = (torch.empty(70, cols + pad, dtype=dtype, device="cuda")[:, :cols] for _ in range(2))
    for into_y, into_total in ((x2, r2), (r2, x2)):
        x2.copy_(x), r2.copy_(res)
        B.pvt_norm_apply(B.make_norm(x2, w, b, residual=r2), y=into_y, total=into_total)
        assert torch.equal(into_y, y) and torch.equal(into_total, total)
    dy, dres = rows(gen, shape, dtype, pad), rows(gen, shape, dtype, pad)
    dx = torch.empty_like(y)
    B.pvt_norm_grad(B.make_norm(total, w), stats, dy, dx, dresidual=dres)
    for at in range(3):
        args = [t.clone(memory_format=torch.preserve_format) if t.is_contiguous() else
                torch.empty(70, cols + pad, dtype=dtype, device="cuda")[:, :cols].copy_(t) for t in (total, dy, dres)]
        B.pvt_norm_grad(B.make_norm(args[0], w), stats, args[1], args[at], dresidual=args[2])
        assert torch.equal(args[at], dx)


def test_rows_with_nan_or_infinity_touch_no_other():
    gen = torch.Generator("cuda").manual_seed(3)
    for cols in (64, 200, 1500, 9000):
        x = torch.randn(40, cols, device="cuda", generator=gen)
        bad = x.clone()
        bad[3, cols // 2], bad[7, 0], bad[39, cols - 1] = math.nan, math.inf, -math.inf
        out, want = torch.empty_like(x), torch.empty_like(x)
        m = B.new_mx(40, cols, B.PVT_MX_E8M0_32)
        B.pvt_norm_apply(B.make_norm(x), y=want)
        B.pvt_norm_apply(B.make_norm(bad), y=out, quantized=m)
        fine = torch.ones(40, dtype=torch.bool, device="cuda")
        fine[[3, 7, 39]] = False
        assert torch.equal(out[fine], want[fine]) and not torch.isfinite(out[~fine]).any()
        check_held(m, out, B.PVT_MX_E8M0_32)


def test_a_constant_row_and_rows_of_zeros():
    x = torch.zeros(3, 777, device="cuda")
    x[1] = 5.0
    w, b = torch.full((777,), 2.0, device="cuda"), torch.full((777,), 0.5, device="cuda")
    y, stats = torch.empty_like(x), torch.empty(3, 2, device="cuda")
    B.pvt_norm_apply(B.make_norm(x, w, b, eps=1e-4), y=y, stats=stats)
    # (a mean of 777 fives rounds: see norm_bounds)
    d_y, _, _ = ref.norm_bounds(x, ref.LAYER, 1e-4, w, b)
    assert ((y.double() - 0.5).abs() <= d_y).all() and (stats[0] == torch.tensor([0.0, 100.0], device="cuda")).all()


def test_rows_beyond_32_bits():
    """A matrix whose last rows lie more than 2^31 elements from its first ones."""
    cols, pitch, n = 256, 1 << 22, 600
    wide = torch.empty(n, pitch, dtype=F16, device="cuda")
    x = wide[:, :cols]
    gen = torch.Generator("cuda").manual_seed(9)
    x.copy_(torch.randn(n, cols, device="cuda", generator=gen))
    y = wide[:, cols:2 * cols]
    stats = torch.empty(n, 2, device="cuda")
    B.pvt_norm_apply(B.make_norm(x), y=y, stats=stats)
    want, _, _ = ref.norm(x, ref.LAYER, 1e-5)
    close(y, want, ref.norm_bounds(x, ref.LAYER, 1e-5)[0], F16)
    dx = wide[:, 2 * cols:3 * cols]
    B.pvt_norm_grad(B.make_norm(x), stats, y, dx)
    close(dx, ref.norm_grad(x, stats, y, ref.LAYER)[0], ref.norm_grad_bounds(x, stats, y, ref.LAYER)[0], F16)


def test_no_result_depends_on_the_run_or_on_what_the_workspace_holds():
    gen = torch.Generator("cuda").manual_seed(4)
    for shape in ((5000, 96), (3000, 1000), (1000, 8192), (300, 30000)):
        x, dy = torch.randn(shape, device="cuda", generator=gen).bfloat16(), torch.randn(shape, device="cuda", generator=gen).bfloat16()
        stats, y = torch.empty(shape[0], 2, device="cuda"), torch.empty_like(x)
        n = B.make_norm(x)
        B.pvt_norm_apply(n, y=y, stats=stats)
        seen = []
        for fill in (0, 0xff, 0x7f):
            ws = B.new_norm_workspace(n).fill_(fill)
            dx, dw, db = torch.empty_like(x), torch.empty(shape[1], device="cuda"), torch.empty(shape[1], device="cuda")
            B.pvt_norm_grad(n, stats, dy, dx, dweight=dw, dbias=db, workspace=ws)
            seen.append((dx, dw, db))
        for other in seen[1:]:
            assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


def test_streams_and_graphs():
    """Calls on a side stream follow it, and a captured step reads what is there when it is replayed."""
    shape = (300, 1000)
    x, res, dy = (torch.empty(shape, dtype=BF16, device="cuda") for _ in range(3))
    w, b = torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    total, y, dx = (torch.empty(shape, dtype=BF16, device="cuda") for _ in range(3))
    stats, dw, db = torch.empty(300, 2, device="cuda"), torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    m = B.new_mx(*shape, B.PVT_MX_E8M0_32)
    fwd, bwd = B.make_norm(x, w, b, residual=res), B.make_norm(total, w)
    ws = B.new_norm_workspace(bwd)
    outs = (total, y, dx, stats, dw, db, m.codes, m.scales)

    def step():
        B.pvt_norm_apply(fwd, y=y, total=total, stats=stats, quantized=m)
        B.pvt_norm_grad(bwd, stats, dy, dx, dresidual=res, dweight=dw, dbias=db, workspace=ws)

    def fill(seed):
        gen = torch.Generator("cuda").manual_seed(seed)
        for t in (x, res, dy, w, b):
            t.copy_(torch.randn(t.shape, device="cuda", generator=gen))
        for t in outs:
            t.fill_(7)

    fill(1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 3):
        fill(seed)
        step()
        want = [t.clone() for t in outs]
        fill(seed)
        graph.replay()
        assert all(torch.equal(a, c) for a, c in zip(outs, want))
        fill(seed)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, c) for a, c in zip(outs, want))


def test_the_workspace_is_checked_and_sized_for_its_shape():
    x, dy = torch.randn(50, 300, device="cuda"), torch.randn(50, 300, device="cuda")
    n = B.make_norm(x)
    stats, dx, dw = torch.empty(50, 2, device="cuda"), torch.full_like(x, 7.0), torch.full((300,), 7.0, device="cuda")
    B.pvt_norm_apply(n, stats=stats)
    ws = B.new_norm_workspace(n)
    for bad, code in ((None, B.PVT_EINVAL), (ws[:-1], B.PVT_EWORKSPACE), (torch.empty(ws.numel() + 16, dtype=torch.uint8, device="cuda")[16:], B.PVT_EINVAL)):
        with pytest.raises(B.PvtError) as e:
            B.pvt_norm_grad(n, stats, dy, dx, dweight=dw, workspace=bad)
        assert e.value.code == code
    assert (dx == 7).all() and (dw == 7).all()


def test_the_binding_refuses_what_does_not_fit():
    x = torch.randn(4, 64, device="cuda")
    n, ws = B.make_norm(x), None
    stats = torch.empty(4, 2, device="cuda")
    for bad in (lambda: B.make_norm(x.cpu()), lambda: B.make_norm(x.double()), lambda: B.make_norm(x[0]),
                lambda: B.make_norm(x, torch.ones(63, device="cuda")), lambda: B.make_norm(x, torch.ones(64)),
                lambda: B.make_norm(x, torch.ones(64, device="cuda"), torch.ones(64, device="cuda").half()),
                lambda: B.make_norm(x, residual=x.half()), lambda: B.make_norm(x, residual=x[:3]),
                lambda: B.make_norm(x[:1].expand(4, 64)), lambda: B.make_norm(torch.randn(64, 4, device="cuda").T),
                lambda: B.pvt_norm_apply(n, y=x.cpu()), lambda: B.pvt_norm_apply(n, y=x[:3]), lambda: B.pvt_norm_apply(n, total=x.half()),
                lambda: B.pvt_norm_apply(n, stats=stats[:3]), lambda: B.pvt_norm_apply(n, quantized=B.new_mx(4, 65, 0)),
                lambda: B.pvt_norm_grad(n, stats, x, x.half()), lambda: B.pvt_norm_grad(n, stats, x, x, dresidual=x.half()),
                lambda: B.pvt_norm_grad(n, stats.double(), x, x), lambda: B.pvt_norm_grad(n, stats, x, x, dweight=x[0].half()),
                lambda: B.pvt_norm_grad(n, stats, x, x, dweight=x[0], dbias=x[0].double())):
        with pytest.raises(ValueError):
            bad()
