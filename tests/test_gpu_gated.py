"""The gated pair of 4-bit products and its gradients against the formulas in float64: few tokens and tiles of 128 and 256, one and
several pairs of blocks to a tile, tile after tile, odd sizes, both formats, all activations, 4-bit results, gradients against
differences, results in the place of operands, graphs, streams, waits that run out, refusals by the binding."""
import math

import pytest
import torch

import block_reference as ref
import student_reference as mx
from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
FORMATS = [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16]
ACTS = [B.PVT_ACT_SILU, B.PVT_ACT_GELU, B.PVT_ACT_GELU_TANH]
# tokens, inputs, outputs
SHAPES = [(1, 1, 1), (1, 33, 8), (2, 256, 129), (3, 1000, 300), (16, 4096, 1000), (5, 600, 5000), (1, 8192, 200), (15, 255, 128),
          (17, 256, 100), (33, 257, 129), (100, 1000, 31), (128, 64, 256), (129, 300, 300), (200, 2048, 1000), (257, 512, 700),
          (300, 100, 4095), (600, 300, 4096), (640, 256, 3700), (1030, 700, 2500), (40, 6200, 500), (300, 7000, 1000), (20, 12300, 200),
          (150, 16000, 640), (700, 96, 128)]


def held(gen, rows, cols, fmt, std, ts=None, pad=0):
    """A 4-bit matrix of random values, and these in float64; rows of codes `pad` bytes further apart than need be."""
    pitch = -(-cols // 32) * 16
    codes = torch.full((rows, pitch + pad), 0xa5, dtype=torch.uint8, device="cuda")[:, :pitch]
    scales = torch.empty(B.pvt_mx_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda")
    scale = torch.tensor([ts], device="cuda") if ts and fmt == B.PVT_MX_E4M3_16 else None
    m = B.make_mx(codes, scales, rows, cols, fmt, tensor_scale=scale)
    B.pvt_mx_quantize(m, std * torch.randn(rows, cols, device="cuda", generator=gen))
    return m, mx.values(*mx.unpack(codes, scales, rows, cols, fmt), fmt, None if scale is None else scale.item())


def operands(case, shape, fmt, same_scale=False):
    gen = torch.Generator("cuda").manual_seed(case)
    tokens, cols, n = shape
    ts = [(None, None, None), (0.002, 0.0005, 0.0005), (None, 0.0005, 0.0007)][case % 3]
    std = 1.5 / math.sqrt(cols)
    x, xv = held(gen, tokens, cols, fmt, 1.0, ts[0], 16 * (case % 2))
    wg, gv = held(gen, n, cols, fmt, std, ts[1], 32 * (case % 2))
    wu, uv = held(gen, n, cols, fmt, std, ts[1] if same_scale else ts[2])
    if same_scale and wu.tensor_scale is not None:
        wu = B.make_mx(wu.codes, wu.scales, n, cols, fmt, tensor_scale=wg.tensor_scale)
    return gen, x, wg, wu, xv, gv, uv


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def close(got, want, bound, dtype):
    slack = bound + ref.rounding(want.abs() + bound, dtype)
    off = (got.double() - want).abs()
    assert (off <= slack).all(), f"off by up to {(off / slack).max().item():.3g} of what is allowed"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case,shape", list(enumerate(SHAPES)))
def test_gated(fmt, case, shape):
    tokens, cols, n = shape
    _, x, wg, wu, xv, gv, uv = operands(case, shape, fmt)
    act, dtype, pad = ACTS[case % 3], TYPES[(case + fmt) % 3], case % 3
    a, b, d_a, d_b = ref.products(xv, gv, uv)
    st = status()
    wide = torch.full((tokens + 1, n + pad), 7.0, dtype=dtype, device="cuda")
    B.pvt_mx_gated(x, wg, wu, h=wide[:-1, :n], activation=act, status=st)
    close(wide[:-1, :n], ref.gated(a, b, act), ref.gated_bound(a, b, d_a, d_b, act), dtype)
    assert (wide[-1] == 7).all() and (wide[:, n:] == 7).all()
    # in 4 bits: those of the binary32 values
    ts = torch.tensor([0.003], device="cuda") if fmt == B.PVT_MX_E4M3_16 and case % 2 else None
    h = torch.empty(tokens, n, device="cuda")
    pitch = -(-n // 32) * 16 + 16
    codes = torch.full((tokens, pitch), 0xa5, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.pvt_mx_scale_bytes(tokens, n, fmt),), 0xa5, dtype=torch.uint8, device="cuda")
    q = B.make_mx(codes, scales, tokens, n, fmt, tensor_scale=ts)
    B.pvt_mx_gated(x, wg, wu, h=h, quantized=q, activation=act, status=st)
    want_codes, want_scales = mx.quantize(h, fmt, None if ts is None else ts.item())
    got_codes, got_scales = mx.unpack(codes, scales, tokens, n, fmt)
    assert torch.equal(got_scales, want_scales) and torch.equal(got_codes, want_codes)
    assert torch.equal(scales, mx.pack(want_codes, want_scales, fmt)[1]) and (codes[:, (n + 1) // 2:] == 0xa5).all()
    assert torch.equal(h.to(dtype), wide[:-1, :n])
    keep = codes.clone(), scales.clone()
    codes.fill_(0xa5), scales.fill_(0xa5)
    B.pvt_mx_gated(x, wg, wu, quantized=q, activation=act, status=st)
    assert torch.equal(codes, keep[0]) and torch.equal(scales, keep[1])
    assert st.item() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case,shape", list(enumerate(SHAPES)))
def test_gradients(fmt, case, shape):
    tokens, cols, n = shape
    gen, x, wg, wu, xv, gv, uv = operands(50 + case, shape, fmt, same_scale=True)
    act, dtype, pad = ACTS[(case + 1) % 3], TYPES[(case + fmt) % 3], case % 3
    a, b, d_a, d_b = ref.products(xv, gv, uv)
    dh = torch.full((tokens, n + pad), math.nan, dtype=dtype, device="cuda")[:, :n]
    dh.copy_(torch.randn(tokens, n, device="cuda", generator=gen))
    pitch = -(-n // 8) * 8 + 8 * (case % 2)
    dgate, dup = (torch.full((tokens + 1, pitch), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    st = status()
    B.pvt_mx_gated_grad(x, wg, wu, dh, dgate[:-1, :n], dup[:-1, :n], activation=act, status=st)
    f, slope = ref.activation(a, act)
    d_gate, d_up = ref.gated_grad_bounds(a, b, d_a, d_b, dh, act)
    close(dgate[:-1, :n], dh.double() * b * slope, d_gate, BF16)
    close(dup[:-1, :n], dh.double() * f, d_up, BF16)
    assert all((t[-1] == 7).all() and (t[:, n:] == 7).all() for t in (dgate, dup))
    # in the place of dh
    if dtype == BF16:
        for at in range(2):
            given = torch.zeros(tokens, pitch, dtype=BF16, device="cuda")[:, :n].copy_(dh)
            other = torch.zeros(tokens, pitch, dtype=BF16, device="cuda")[:, :n]
            B.pvt_mx_gated_grad(x, wg, wu, given, *((given, other) if at == 0 else (other, given)), activation=act, status=st)
            assert torch.equal(given if at == 0 else other, dgate[:-1, :n]) and torch.equal(other if at == 0 else given, dup[:-1, :n])
    # by the input, exactly from what was written
    dg, du = dgate[:-1, :n], dup[:-1, :n]
    want = dg.double() @ gv + du.double() @ uv
    off = (2 * n + 4) * 2.0 ** -23 * (dg.double().abs() @ gv.abs() + du.double().abs() @ uv.abs())
    for out in TYPES:
        dx = torch.full((tokens + 1, cols + pad), 7.0, dtype=out, device="cuda")
        B.pvt_mx_gated_grad_input(dg, du, wg, wu, dx[:-1, :cols], status=st)
        close(dx[:-1, :cols], want, off, out)
        assert (dx[-1] == 7).all() and (dx[:, cols:] == 7).all()
    assert st.item() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens,cols,n", [(1, 257, 2050), (129, 512, 1024), (130, 4096, 700), (200, 300, 9000), (256, 1024, 2048), (300, 1030, 1500),
                                           (520, 768, 4096), (700, 2049, 333)])
def test_input_gradient_by_any_number_of_blocks(tokens, cols, n, fmt):
    """Tiles whose steps single blocks or pairs of blocks share, ragged in every direction; the same bits each time."""
    gen = torch.Generator("cuda").manual_seed(tokens + n)
    wg, gv = held(gen, n, cols, fmt, 0.1)
    wu, uv = held(gen, n, cols, fmt, 0.1)
    pitch = -(-n // 8) * 8
    dg, du = (torch.randn(tokens, pitch, device="cuda", generator=gen).bfloat16()[:, :n] for _ in range(2))
    want = dg.double() @ gv + du.double() @ uv
    off = (2 * n + 4) * 2.0 ** -23 * (dg.double().abs() @ gv.abs() + du.double().abs() @ uv.abs())
    outs = []
    st = status()
    for _ in range(2):
        dx = torch.full((tokens + 1, cols + 3), 7.0, device="cuda")
        B.pvt_mx_gated_grad_input(dg, du, wg, wu, dx[:-1, :cols], status=st)
        outs.append(dx)
    close(outs[0][:-1, :cols], want, off, torch.float32)
    assert (outs[0][-1] == 7).all() and (outs[0][:, cols:] == 7).all()
    assert torch.equal(outs[0], outs[1]) and st.item() == 0


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """f' is the derivative of f, and the kernel's gradients are those of sum(dh h) by a and b."""
    a = torch.linspace(-8, 8, 2001, dtype=torch.float64)
    f, slope = ref.activation(a, act)
    h = 1e-5
    assert ((ref.activation(a + h, act)[0] - ref.activation(a - h, act)[0]) / (2 * h) - slope).abs().max() <= 1e-9
    assert slope.abs().max() <= 1.13 and ((ref.activation(a + h, act)[1] - ref.activation(a - h, act)[1]) / (2 * h)).abs().max() <= 1.0
    gen = torch.Generator("cuda").manual_seed(3)
    x, xv = held(gen, 20, 64, B.PVT_MX_E8M0_32, 1.0)
    wg, gv = held(gen, 40, 64, B.PVT_MX_E8M0_32, 0.2)
    wu, uv = held(gen, 40, 64, B.PVT_MX_E8M0_32, 0.2)
    dh = torch.randn(20, 40, device="cuda", generator=gen)
    dgate, dup = (torch.empty(20, 40, dtype=BF16, device="cuda") for _ in range(2))
    B.pvt_mx_gated_grad(x, wg, wu, dh, dgate, dup, activation=act)
    a, b = xv @ gv.T, xv @ uv.T
    by_a = dh * (ref.gated(a + h, b, act) - ref.gated(a - h, b, act)) / (2 * h)
    by_b = dh * (ref.gated(a, b + h, act) - ref.gated(a, b - h, act)) / (2 * h)
    # half a step of bfloat16, and 1e-5 for everything in binary32 and the differences
    assert ((dgate - by_a).abs() <= 2.0 ** -8 * by_a.abs() + 1e-5).all() and ((dup - by_b).abs() <= 2.0 ** -8 * by_b.abs() + 1e-5).all()


@pytest.mark.parametrize("tokens", [5, 40, 300])
@pytest.mark.parametrize("act", ACTS)
def test_large_and_small_products(tokens, act):
    """Activations far from 0 on both sides: 0 or the product itself, never a NaN."""
    x, w = torch.zeros(tokens, 64, device="cuda"), torch.zeros(200, 64, device="cuda")
    x[:, 0] = 1.0
    w[:, 0] = torch.tensor([0.0, 1.0, -1.0, 96.0, -96.0, 2.0 ** 14, -2.0 ** 14, 1.5]).cuda().repeat(25)
    xm, wm = B.new_mx(tokens, 64, B.PVT_MX_E8M0_32), B.new_mx(200, 64, B.PVT_MX_E8M0_32)
    B.pvt_mx_quantize(xm, x), B.pvt_mx_quantize(wm, w)
    h, dh = torch.empty(tokens, 200, device="cuda"), torch.ones(tokens, 200, device="cuda")
    dgate, dup = (torch.empty(tokens, 200, dtype=BF16, device="cuda") for _ in range(2))
    B.pvt_mx_gated(xm, wm, wm, h=h, activation=act)
    B.pvt_mx_gated_grad(xm, wm, wm, dh, dgate, dup, activation=act)
    a = (x @ w.T).double()
    f, slope = ref.activation(a, act)
    zero = torch.zeros_like(a)
    close(h, f * a, ref.gated_bound(a, a, zero, zero, act), F32)
    d_gate, d_up = ref.gated_grad_bounds(a, a, zero, zero, dh, act)
    close(dgate, a * slope, d_gate, BF16)
    close(dup, f, d_up, BF16)


@pytest.mark.parametrize("tokens", [5, 40])
@pytest.mark.parametrize("act", ACTS)
def test_products_beyond_where_cubes_are_numbers(tokens, act):
    """f' of a huge product is 0 or 1, where a^2 or a^3 is infinite in binary32 too."""
    x, w = torch.zeros(tokens, 64, device="cuda"), torch.zeros(64, 64, device="cuda")
    x[:, 0] = 2.0 ** 40
    w[:, 0] = torch.tensor([2.0 ** 10, -2.0 ** 10, 2.0 ** 50, -2.0 ** 50, 2.0 ** 80, -2.0 ** 80, 0.0, 1.0]).cuda().repeat(8)
    xm, wm, one = B.new_mx(tokens, 64, B.PVT_MX_E8M0_32), B.new_mx(64, 64, B.PVT_MX_E8M0_32), B.new_mx(64, 64, B.PVT_MX_E8M0_32)
    B.pvt_mx_quantize(xm, x), B.pvt_mx_quantize(wm, w), B.pvt_mx_quantize(one, (w != 5) * torch.eye(1, 64, device="cuda") * 2.0 ** -40)
    h, dh = torch.empty(tokens, 64, device="cuda"), torch.ones(tokens, 64, device="cuda")
    dgate, dup = (torch.empty(tokens, 64, dtype=BF16, device="cuda") for _ in range(2))
    B.pvt_mx_gated(xm, wm, one, h=h, activation=act)
    B.pvt_mx_gated_grad(xm, wm, one, dh, dgate, dup, activation=act)
    a = x @ w.T
    want = torch.where(a > 0, a, torch.zeros_like(a))  # (a product with the other matrix of 1)
    assert torch.equal(h, want) and torch.equal(dup, want.bfloat16())
    slope = torch.where(a > 0, torch.ones_like(a), torch.where(a < 0, torch.zeros_like(a), torch.full_like(a, 0.5)))
    assert torch.equal(dgate, slope.bfloat16())


@pytest.mark.parametrize("tokens", [7, 60, 300])
def test_what_is_not_a_number_stays_in_its_token_and_output(tokens):
    gen = torch.Generator("cuda").manual_seed(tokens)
    x, w = torch.randn(tokens, 512, device="cuda", generator=gen), 0.05 * torch.randn(300, 512, device="cuda", generator=gen)
    bad_x, bad_w = x.clone(), w.clone()
    bad_x[2, 100], bad_w[150, 3] = math.nan, math.inf
    m = [B.new_mx(t.shape[0], 512, B.PVT_MX_E8M0_32) for t in (x, w, bad_x, bad_w)]
    for held_, t in zip(m, (x, w, bad_x, bad_w)):
        B.pvt_mx_quantize(held_, t)
    want, got = torch.empty(tokens, 300, device="cuda"), torch.empty(tokens, 300, device="cuda")
    q = B.new_mx(tokens, 300, B.PVT_MX_E8M0_32)
    B.pvt_mx_gated(m[0], m[1], m[1], h=want)
    B.pvt_mx_gated(m[2], m[1], m[3], h=got, quantized=q)
    gone = torch.zeros_like(got, dtype=torch.bool)
    gone[2], gone[:, 150] = True, True
    assert torch.isnan(got[gone]).all() and torch.equal(got[~gone], want[~gone])
    codes, scales = mx.quantize(got, B.PVT_MX_E8M0_32)
    assert torch.equal(q.scales, mx.pack(codes, scales, B.PVT_MX_E8M0_32)[1])


def test_results_do_not_depend_on_the_run_and_graphs_read_what_is_there():
    for shape, fmt in (((9, 4096, 3000), 0), ((300, 2048, 4096), 1), ((64, 8192, 704), 0)):
        tokens, cols, n = shape
        gen = torch.Generator("cuda").manual_seed(1)
        x, wg, wu = B.new_mx(tokens, cols, fmt), B.new_mx(n, cols, fmt), B.new_mx(n, cols, fmt)
        h, q = torch.empty(tokens, n, dtype=BF16, device="cuda"), B.new_mx(tokens, n, fmt)
        dh, dgate, dup = (torch.empty(tokens, n, dtype=BF16, device="cuda") for _ in range(3))
        dx, st = torch.empty(tokens, cols, device="cuda"), status()

        def step():
            B.pvt_mx_gated(x, wg, wu, h=h, quantized=q, status=st)
            B.pvt_mx_gated_grad(x, wg, wu, dh, dgate, dup, status=st)
            B.pvt_mx_gated_grad_input(dgate, dup, wg, wu, dx, status=st)

        def fill(seed):
            gen.manual_seed(seed)
            for m in (x, wg, wu):
                B.pvt_mx_quantize(m, torch.randn(m.rows, cols, device="cuda", generator=gen) * (1.0 if m is x else 0.02))
            dh.copy_(torch.randn(tokens, n, device="cuda", generator=gen))
            for t in (h, q.codes, q.scales, dgate, dup, dx):
                t.fill_(7)

        outs = lambda: [t.clone() for t in (h, q.codes, q.scales, dgate, dup, dx)]  # noqa: E731
        fill(1)
        step()
        first = outs()
        fill(1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, r) for p, r in zip(first, outs()))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        fill(2)
        step()
        want = outs()
        fill(2)
        graph.replay()
        assert all(torch.equal(p, r) for p, r in zip(want, outs())) and st.item() == 0


def test_two_calls_at_once():
    """Calls on two streams have nothing in common that they write."""
    gen = torch.Generator("cuda").manual_seed(8)
    sets = []
    for tokens, cols, n in ((1, 4096, 2000), (500, 1024, 3000)):
        x, _ = held(gen, tokens, cols, 0, 1.0)
        wg, _ = held(gen, n, cols, 0, 0.02)
        wu, _ = held(gen, n, cols, 0, 0.02)
        want = torch.empty(tokens, n, dtype=BF16, device="cuda")
        B.pvt_mx_gated(x, wg, wu, h=want)
        sets.append((x, wg, wu, want, [torch.empty_like(want) for _ in range(20)]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for i in range(20):
        for s, (x, wg, wu, _, outs) in zip(streams, sets):
            B.pvt_mx_gated(x, wg, wu, h=outs[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for *_, want, outs in sets for o in outs)


@pytest.mark.parametrize("tokens,withhold", [(3, 0), (3, 2), (200, 0), (200, 5), (600, 3)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_correct(tokens, withhold):
    """The bound of the on-chip waits is lowered and every block leaves out one copy; see the test of the search kernels' waits."""
    gen = torch.Generator("cuda").manual_seed(tokens)
    x, xv = held(gen, tokens, 4096, 0, 1.0)
    wg, gv = held(gen, 2000, 4096, 0, 0.02)
    wu, uv = held(gen, 2000, 4096, 0, 0.02)
    h, dh = torch.empty(tokens, 2000, device="cuda"), torch.ones(tokens, 2000, device="cuda")
    dgate, dup = (torch.empty(tokens, 2000, dtype=BF16, device="cuda") for _ in range(2))
    dx = torch.empty(tokens, 4096, device="cuda")
    calls = (lambda st: B.pvt_mx_gated(x, wg, wu, h=h, status=st), lambda st: B.pvt_mx_gated_grad(x, wg, wu, dh, dgate, dup, status=st),
             lambda st: B.pvt_mx_gated_grad_input(dgate, dup, wg, wu, dx, status=st))
    for call in calls:
        st = status()
        B.pvt_test_wait_limit(20000, withhold)
        try:
            call(st)
            torch.cuda.synchronize()
        finally:
            B.pvt_test_wait_limit(0, -1)
        assert st.item() & B.PVT_DEV_WAIT_EXPIRED
    st = status()
    for call in calls:
        call(st)
    a, b, d_a, d_b = ref.products(xv, gv, uv)
    close(h, ref.gated(a, b, 0), ref.gated_bound(a, b, d_a, d_b, 0), F32)
    want = dgate.double() @ gv + dup.double() @ uv
    close(dx, want, 4004 * 2.0 ** -23 * (dgate.double().abs() @ gv.abs() + dup.double().abs() @ uv.abs()), F32)
    assert st.item() == 0


def test_the_binding_refuses_what_does_not_fit():
    x, w, other = B.new_mx(4, 64, 0), B.new_mx(24, 64, 0), B.new_mx(25, 64, 0)
    h, d = torch.empty(4, 24, device="cuda"), torch.empty(4, 24, dtype=BF16, device="cuda")
    for bad in (lambda: B.pvt_mx_gated(x, w, w, h=h.cpu()), lambda: B.pvt_mx_gated(x, w, w, h=h[:3]), lambda: B.pvt_mx_gated(x, w, w, h=h.double()),
                lambda: B.pvt_mx_gated(x, w, w, quantized=B.new_mx(4, 25, 0)), lambda: B.pvt_mx_gated(x, w, w, quantized=B.new_mx(4, 24, 1)),
                lambda: B.pvt_mx_gated_grad(x, w, w, h, h, d), lambda: B.pvt_mx_gated_grad(x, w, w, h[:3], d, d.clone()),
                lambda: B.pvt_mx_gated_grad(x, w, w, h, d, torch.empty(4, 32, dtype=BF16, device="cuda")[:, :24]),
                lambda: B.pvt_mx_gated_grad_input(d, h, w, w, torch.empty(4, 64, device="cuda")),
                lambda: B.pvt_mx_gated_grad_input(d, d, w, w, h)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.pvt_mx_gated(x, w, other, h=h), lambda: B.pvt_mx_gated(x, w, w), lambda: B.pvt_mx_gated(x, w, w, h=h, activation=3),
                lambda: B.pvt_mx_gated_grad(x, w, w, h, d, d), lambda: B.pvt_mx_gated_grad_input(d, d, w, other, torch.empty(4, 64, device="cuda"))):
        with pytest.raises(B.PvtError) as e:
            bad()
        assert e.value.code == B.PVT_EINVAL
