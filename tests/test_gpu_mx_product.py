"""Products of matrices in 4-bit block floating point and their gradients, against float64.

Most inputs are drawn so that every partial sum is a whole multiple of a power of two below 2^24 times it: binary32 holds each of
them, whatever the order, so results have to be equal to the last bit (and then rounded once where they are 16-bit)."""
import math

import pytest
import torch

import student_reference as ref
from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

FORMATS = [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16]


def held(rows, cols, fmt, seed, scales=None, tensor_scale=None, fill=0xff):
    """A random matrix in its bytes, and its float64 values; scales between 1/2 and 2 unless given."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 16, (rows, cols), device="cuda", generator=gen)
    if scales is None:
        some = torch.tensor([126, 127, 128] if fmt == B.PVT_MX_E8M0_32 else [48, 52, 56, 60, 64], device="cuda")
        pick = torch.randint(0, len(some), (rows, -(-cols // ref.BLOCK[fmt])), device="cuda", generator=gen)
        scales = some[pick]
    # (whatever lies behind a row's last code must not matter)
    h, s = ref.pack(codes, scales, fmt, fill=fill)
    ts = None if tensor_scale is None else torch.tensor([tensor_scale], dtype=torch.float32, device="cuda")
    return B.make_mx(h, s, rows, cols, fmt, tensor_scale=ts), ref.values(codes, scales, fmt)


SHAPES = [  # tokens, inputs, outputs
    (1, 1, 1), (1, 32, 16), (1, 4096, 129), (2, 257, 128), (7, 1000, 300), (16, 512, 2048), (17, 255, 127), (33, 300, 64),
    (64, 2049, 640), (65, 256, 500), (128, 768, 128), (129, 513, 257), (256, 1024, 256), (257, 640, 384), (300, 33, 1000),
    (513, 1537, 130), (1100, 520, 4200), (20, 6200, 500), (140, 12300, 300), (260, 7000, 2100),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens,inputs,outputs", SHAPES)
def test_product_is_exact_where_binary32_is(tokens, inputs, outputs, fmt):
    x, xv = held(tokens, inputs, fmt, 1)
    w, wv = held(outputs, inputs, fmt, 2)
    want = xv @ wv.T
    assert want.abs().max() < 2 ** 24 / 64  # multiples of 1/64
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        y = torch.full((tokens, outputs), math.nan, dtype=dtype, device="cuda")
        B.pvt_mx_product(x, w, y, status=status)
        assert torch.equal(y, want.float().to(dtype))
    assert status.item() == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_product_into_a_part_of_a_wider_matrix(fmt):
    x, xv = held(20, 400, fmt, 3)
    w, wv = held(77, 400, fmt, 4)
    wide = torch.full((20, 100), 5.0, device="cuda")
    B.pvt_mx_product(x, w, wide[:, 11:88])
    assert torch.equal(wide[:, 11:88], (xv @ wv.T).float())
    assert (wide[:, :11] == 5).all() and (wide[:, 88:] == 5).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens", [1, 100, 300])
def test_product_of_numbers_as_they_come(tokens, fmt):
    """Each of the sum's additions is off by at most 2^-23 of a partial sum, which sum |x w| bounds: inputs * 2^-23 of that."""
    inputs, outputs = 3000, 700
    gen = torch.Generator(device="cuda").manual_seed(9)
    ts = [0.0031, 0.00017] if fmt == B.PVT_MX_E4M3_16 else [None, None]
    ms, vs = [], []
    for rows, scale in ((tokens, ts[0]), (outputs, ts[1])):
        x = torch.randn(rows, inputs, device="cuda", generator=gen)
        t = None if scale is None else torch.tensor([scale], dtype=torch.float32, device="cuda")
        m = B.new_mx(rows, inputs, fmt, tensor_scale=t)
        B.pvt_mx_quantize(m, x)
        codes, scales = ref.unpack(m.codes, m.scales, rows, inputs, fmt)
        ms.append(m)
        vs.append(ref.values(codes, scales, fmt, None if t is None else t.item()))
    y = torch.empty(tokens, outputs, device="cuda")
    B.pvt_mx_product(ms[0], ms[1], y)
    bound = (inputs + 4) * 2.0 ** -23 * (vs[0].abs() @ vs[1].abs().T)
    assert ((y.double() - vs[0] @ vs[1].T).abs() <= bound).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_scales_over_their_whole_range(fmt):
    """One block of each row at its own scale: a product of two is exact whatever the scales, as long as binary32 holds it."""
    rows, cols = 130, ref.BLOCK[fmt]
    scales = (torch.arange(rows, device="cuda")[:, None] % 120 + 4 if fmt == B.PVT_MX_E4M3_16
              else torch.arange(rows, device="cuda")[:, None] + 62)
    w, wv = held(rows, cols, fmt, 5, scales=scales)
    x, xv = held(3, cols, fmt, 6)
    y = torch.empty(3, rows, device="cuda")
    B.pvt_mx_product(x, w, y)
    assert torch.equal(y, (xv @ wv.T).float())


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_nan_scale_reaches_its_own_results_only(fmt):
    b = ref.BLOCK[fmt]
    scales = torch.full((200, 20), 127 if fmt == B.PVT_MX_E8M0_32 else 56, device="cuda")
    scales[150, 7] = 255 if fmt == B.PVT_MX_E8M0_32 else 127
    w, wv = held(200, 20 * b, fmt, 7, scales=scales)
    x, xv = held(5, 20 * b, fmt, 8)
    y = torch.empty(5, 200, device="cuda")
    B.pvt_mx_product(x, w, y)
    assert torch.isnan(y[:, 150]).all()
    keep = [i for i in range(200) if i != 150]
    assert torch.equal(y[:, keep], (xv @ wv[keep].T).float())
    dy = torch.ones(5, 200, dtype=torch.bfloat16, device="cuda")
    dx = torch.empty(5, 20 * b, device="cuda")
    B.pvt_mx_grad_input(dy, w, dx)
    assert torch.isnan(dx[:, 7 * b:8 * b]).all() and not torch.isnan(dx[:, :7 * b]).any() and not torch.isnan(dx[:, 8 * b:]).any()


def gradient(tokens, outputs, seed):
    """Small whole numbers, rows a multiple of 8 elements apart, NaN beside them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((tokens, -(-outputs // 8) * 8 + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :outputs] = torch.randint(-4, 5, (tokens, outputs), device="cuda", generator=gen).bfloat16()
    return wide[:, :outputs]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens,inputs,outputs", SHAPES + [(700, 4100, 3000), (2048, 300, 5000)])
def test_gradients_are_exact_where_binary32_is(tokens, inputs, outputs, fmt):
    x, xv = held(tokens, inputs, fmt, 11)
    w, wv = held(outputs, inputs, fmt, 12)
    dy = gradient(tokens, outputs, 13)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = dy.double() @ wv
    assert want.abs().max() < 2 ** 24 / 16
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        dx = torch.full((tokens, inputs), math.nan, dtype=dtype, device="cuda")
        B.pvt_mx_grad_input(dy, w, dx, status=status)
        assert torch.equal(dx, want.float().to(dtype))
    want = dy.double().T @ xv
    assert want.abs().max() < 2 ** 24 / 16
    dw = torch.full((outputs, inputs), math.nan, device="cuda")
    B.pvt_mx_grad_weight(dy, x, dw, status=status)
    assert torch.equal(dw, want.float())
    B.pvt_mx_grad_weight(dy, x, dw, accumulate=True, status=status)
    assert torch.equal(dw, 2 * want.float())
    assert status.item() == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_gradients_of_numbers_as_they_come(fmt):
    """As for the product: sums of n terms within n * 2^-23 of the sum of magnitudes, and one rounding of the result."""
    tokens, inputs, outputs = 333, 900, 1200
    gen = torch.Generator(device="cuda").manual_seed(21)
    ts = 0.0023 if fmt == B.PVT_MX_E4M3_16 else None
    t = None if ts is None else torch.tensor([ts], dtype=torch.float32, device="cuda")
    dy = torch.randn(tokens, outputs, device="cuda", generator=gen).bfloat16()
    for rows, transposed in ((outputs, False), (tokens, True)):
        m = B.new_mx(rows, inputs, fmt, tensor_scale=t)
        B.pvt_mx_quantize(m, torch.randn(rows, inputs, device="cuda", generator=gen))
        v = ref.values(*ref.unpack(m.codes, m.scales, rows, inputs, fmt), fmt, None if t is None else t.item())
        a = dy.double().T if transposed else dy.double()
        out = torch.empty(a.shape[0], inputs, device="cuda")
        if transposed:
            B.pvt_mx_grad_weight(dy, m, out)
        else:
            B.pvt_mx_grad_input(dy, m, out)
        assert ((out.double() - a @ v).abs() <= (rows + 4) * 2.0 ** -23 * (a.abs() @ v.abs())).all()


@pytest.mark.parametrize("byte", [0, 1, 100, 200, 250])
def test_gradients_under_far_scales(byte):
    """Elements under scales far from 1 stay exact in bfloat16, those without a leading one included."""
    scales = torch.full((4, 2), byte, device="cuda")
    w, wv = held(4, 64, B.PVT_MX_E8M0_32, 14, scales=scales)
    dy = torch.zeros(4, 4, dtype=torch.bfloat16, device="cuda")
    dy.fill_diagonal_(0.5)
    wide = torch.zeros(4, 8, dtype=torch.bfloat16, device="cuda")
    wide[:, :4] = dy
    dx = torch.empty(4, 64, device="cuda")
    B.pvt_mx_grad_input(wide[:, :4], w, dx)
    want = (0.5 * wv).float()
    # binary32 sums may leave out numbers below 2^-126; nothing else may be lost
    assert torch.equal(torch.where(want.abs() < 2.0 ** -126, 0.0, dx), torch.where(want.abs() < 2.0 ** -126, 0.0, want))
    assert (dx[want.abs() < 2.0 ** -126].abs() < 2.0 ** -126).all()


def test_calls_repeat_to_the_last_bit():
    x, _ = held(40, 5000, B.PVT_MX_E4M3_16, 15, tensor_scale=0.37)
    w, _ = held(900, 5000, B.PVT_MX_E4M3_16, 16, tensor_scale=0.11)
    dy = torch.randn(40, 904, device="cuda").bfloat16()[:, :900]
    first = None
    for _ in range(5):
        y, dx, dw = torch.empty(40, 900, device="cuda"), torch.empty(40, 5000, device="cuda"), torch.empty(900, 5000, device="cuda")
        B.pvt_mx_product(x, w, y)
        B.pvt_mx_grad_input(dy, w, dx)
        B.pvt_mx_grad_weight(dy, x, dw)
        now = (y, dx, dw)
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now


def test_captured_calls_and_another_stream():
    x, xv = held(9, 700, B.PVT_MX_E8M0_32, 17)
    w, wv = held(300, 700, B.PVT_MX_E8M0_32, 18)
    y = torch.zeros(9, 300, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.pvt_mx_product(x, w, y)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, (xv @ wv.T).float())
    graph = torch.cuda.CUDAGraph()
    source = torch.randn(9, 700, device="cuda")
    v = torch.zeros(9, 700, device="cuda")
    with torch.cuda.graph(graph):
        B.pvt_mx_quantize(x, source)
        B.pvt_mx_product(x, w, y)
        B.pvt_mx_dequant(x, v)
    for seed in (1, 2):
        source.copy_(torch.randn(9, 700, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        codes, scales = ref.quantize(source, B.PVT_MX_E8M0_32)
        now = ref.values(codes, scales, B.PVT_MX_E8M0_32)
        assert torch.equal(v, now.float())
        assert ((y.double() - now @ wv.T).abs() <= 704 * 2.0 ** -23 * (now.abs() @ wv.abs().T)).all()


@pytest.mark.parametrize("tokens", [40, 1300])
@pytest.mark.parametrize("what", ["product", "input", "weight"])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_correct(what, tokens):
    x, xv = held(tokens, 3000, B.PVT_MX_E8M0_32, 19)
    w, wv = held(2000, 3000, B.PVT_MX_E8M0_32, 20)
    dy = gradient(tokens, 2000, 23)
    out = {"product": torch.empty(tokens, 2000, device="cuda"), "input": torch.empty(tokens, 3000, device="cuda"),
           "weight": torch.empty(2000, 3000, device="cuda")}[what]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        if what == "product":
            B.pvt_mx_product(x, w, out, status=status)
        elif what == "input":
            B.pvt_mx_grad_input(dy, w, out, status=status)
        else:
            B.pvt_mx_grad_weight(dy, x, out, status=status)

    B.pvt_test_wait_limit(20000, 0)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        B.pvt_test_wait_limit(0, -1)
    assert status.item() & B.PVT_DEV_WAIT_EXPIRED
    status.zero_()
    call()
    assert status.item() == 0
    want = {"product": xv @ wv.T, "input": dy.double() @ wv, "weight": dy.double().T @ xv}[what]
    assert torch.equal(out, want.float())


@pytest.mark.parametrize("tokens", [5, 200, 600])
@pytest.mark.parametrize("one,other", [(1e25, 1e25), (1e-25, 1e-25), (1e30, 1e-30), (1e-44, 1e4), (3e38, 1.0), (1.0, 1e-41)])
def test_tensor_scales_whose_product_is_no_number(one, other, tokens):
    """Both roundings of the result are half a step each: 2^-22 of it in all, and half of the smallest number."""
    fmt = B.PVT_MX_E4M3_16
    x, xv = held(tokens, 80, fmt, 31, tensor_scale=one)
    w, wv = held(704, 80, fmt, 32, tensor_scale=other)
    x.codes[:3] = 0
    xv[:3] = 0

    def agree(got, sums, *scales):
        # (scaled after the sums, which are exact: scaled terms would not cancel)
        want = sums * math.prod(s.tensor_scale.item() for s in scales)
        rounded = want.float().double()
        near = (got.double() - want).abs() <= want.abs() * 2.0 ** -22 + 2.0 ** -149
        return bool((near | (got.double() == rounded)).all())

    y = torch.empty(tokens, 704, device="cuda")
    B.pvt_mx_product(x, w, y)
    assert agree(y, xv @ wv.T, x, w) and (y[:3] == 0).all()
    dy = gradient(tokens, 704, 33) * 2.0 ** -20
    dy[:2] = 0
    dx = torch.empty(tokens, 80, device="cuda")
    B.pvt_mx_grad_input(dy, w, dx)
    assert agree(dx, dy.double() @ wv, w) and (dx[:2] == 0).all()
    dw = torch.empty(704, 80, device="cuda")
    B.pvt_mx_grad_weight(dy, x, dw)
    assert agree(dw, dy.double().T @ xv, x)


def test_calls_on_several_streams_at_once():
    """Products and gradients of few and many tiles side by side: each takes tensor memory for itself, and results are those of
    the same calls alone."""
    jobs = []
    for i, (tokens, inputs, outputs) in enumerate([(4, 2048, 4096), (600, 1024, 2048), (40, 3000, 1500), (1100, 700, 3000)]):
        fmt = FORMATS[i % 2]
        x, _ = held(tokens, inputs, fmt, 40 + i)
        w, _ = held(outputs, inputs, fmt, 50 + i)
        dy = gradient(tokens, outputs, 60 + i)
        outs = [torch.empty(tokens, outputs, device="cuda"), torch.empty(tokens, inputs, device="cuda"),
                torch.empty(outputs, inputs, device="cuda")]

        def run(x=x, w=w, dy=dy, outs=outs):
            B.pvt_mx_product(x, w, outs[0])
            B.pvt_mx_grad_input(dy, w, outs[1])
            B.pvt_mx_grad_weight(dy, x, outs[2])
        run()
        jobs.append((run, outs, [o.clone() for o in outs]))
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, (run, outs, _) in zip(streams, jobs):
            with torch.cuda.stream(stream):
                for o in outs:
                    o.fill_(math.nan)
                run()
    torch.cuda.synchronize()
    for _, outs, want in jobs:
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("tokens,inputs,outputs", [(40, 12300, 300), (3, 6000, 200)])
def test_a_wait_that_runs_out_in_blocks_that_share_a_tile(tokens, inputs, outputs):
    """All blocks of a cluster come to its barriers, whatever one of them has given up."""
    x, xv = held(tokens, inputs, B.PVT_MX_E8M0_32, 71)
    w, wv = held(outputs, inputs, B.PVT_MX_E8M0_32, 72)
    y = torch.empty(tokens, outputs, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pvt_test_wait_limit(20000, 1)
    try:
        B.pvt_mx_product(x, w, y, status=status)
        torch.cuda.synchronize()
    finally:
        B.pvt_test_wait_limit(0, -1)
    assert status.item() & B.PVT_DEV_WAIT_EXPIRED
    status.zero_()
    B.pvt_mx_product(x, w, y, status=status)
    assert status.item() == 0 and torch.equal(y, (xv @ wv.T).float())
