"""The feed-forward half of a block through its calls one after the other, forward, backward and the steps that follow: every stage from
its definition and what the stage ahead has written, gradients added up over batches, the norm's weights by Adam, the layers by the V step."""
import math

import numpy as np
import pytest
import torch

import block_reference as block
import student_reference as mx
from oracle import pvt_oracle as oracle
from paper_2405_14852_b200 import binding as B
from paper_2405_14852_b200 import synth
from paper_2405_14852_b200.vstep import FeedForward, VStepLayer

pytestmark = pytest.mark.gpu

WIDTH, INNER = 256, 704


def layers(scale=0.05):
    made = []
    for i, (rows, cols) in enumerate(((INNER, WIDTH), (INNER, WIDTH), (WIDTH, INNER))):
        L = synth.make_layer(rows, cols, cfg=80 + i, codebook_size=256, codebook_fp16=True)
        made.append(VStepLayer.from_host(L))
        made[-1].scale.mul_(scale / made[-1].dequant().std())
        made[-1].W.copy_(made[-1].dequant())
    return made


def values(m):
    ts = None if m.tensor_scale is None else m.tensor_scale.item()
    return mx.values(*mx.unpack(m.codes, m.scales, m.rows, m.cols, m.format), m.format, ts)


def within(got, want, bound, dtype=torch.float32):
    slack = bound + block.rounding(want.abs() + bound, dtype)
    off = (got.double() - want).abs()
    assert (off <= slack).all(), f"off by up to {(off / slack).max().item():.3g} of what is allowed"


def sums(terms, a, b):
    """a @ b and how far a binary32 sum of so many terms may be off"""
    return a @ b, (terms + 4) * 2.0 ** -23 * (a.abs() @ b.abs())


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("tokens,kind,act", [(1, B.PVT_NORM_RMS, B.PVT_ACT_SILU), (40, B.PVT_NORM_LAYER, B.PVT_ACT_GELU),
                                             (333, B.PVT_NORM_RMS, B.PVT_ACT_GELU_TANH)])
def test_every_stage_from_the_one_ahead(fmt, tokens, kind, act):
    gen = torch.Generator("cuda").manual_seed(tokens)
    gate, up, down = layers()
    weight = 1 + 0.2 * torch.randn(WIDTH, device="cuda", generator=gen)
    bias = 0.1 * torch.randn(WIDTH, device="cuda", generator=gen) if kind == B.PVT_NORM_LAYER else None
    ff = FeedForward(gate, up, down, weight, bias, kind=kind, activation=act, fmt=fmt)
    x, residual = (torch.randn(tokens, WIDTH, device="cuda", generator=gen).bfloat16() for _ in range(2))
    y, total = ff.forward(x, residual)
    assert torch.equal(total, (x.float() + residual.float()).bfloat16())
    assert ff.w_gate.tensor_scale is ff.w_up.tensor_scale
    _, stats, xq, hq = ff._kept
    # the 4-bit operands are those of binary32 results within their bounds
    n32 = torch.empty(tokens, WIDTH, device="cuda")
    B.pvt_norm_apply(B.make_norm(total, weight, bias, kind=kind), y=n32)
    within(n32, block.norm(total, kind, 1e-5, weight, bias)[0], block.norm_bounds(total, kind, 1e-5, weight, bias)[0])
    codes, scales = mx.quantize(n32, fmt)
    assert torch.equal(xq.scales, mx.pack(codes, scales, fmt)[1]) and torch.equal(mx.unpack(xq.codes, xq.scales, tokens, WIDTH, fmt)[0], codes)
    xv, gv, uv, dv = values(xq), values(ff.w_gate), values(ff.w_up), values(ff.w_down)
    h32 = torch.empty(tokens, INNER, device="cuda")
    B.pvt_mx_gated(xq, ff.w_gate, ff.w_up, h=h32, activation=act)
    a, b, d_a, d_b = block.products(xv, gv, uv)
    within(h32, block.gated(a, b, act), block.gated_bound(a, b, d_a, d_b, act))
    codes, scales = mx.quantize(h32, fmt)
    assert torch.equal(hq.scales, mx.pack(codes, scales, fmt)[1]) and torch.equal(mx.unpack(hq.codes, hq.scales, tokens, INNER, fmt)[0], codes)
    hv = values(hq)
    within(y, *sums(INNER, hv, dv.T), torch.bfloat16)

    dy, dtotal = (torch.randn(tokens, WIDTH, device="cuda", generator=gen).bfloat16() for _ in range(2))
    dx = ff.backward(dy, dtotal, first=True)
    dh, dgate, dup = (torch.empty(tokens, INNER, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    dn = torch.empty(tokens, WIDTH, dtype=torch.bfloat16, device="cuda")
    B.pvt_mx_grad_input(dy, ff.w_down, dh)
    within(dh, *sums(WIDTH, dy.double(), dv), torch.bfloat16)
    within(down.g, *sums(tokens, dy.double().T, hv))
    B.pvt_mx_gated_grad(xq, ff.w_gate, ff.w_up, dh, dgate, dup, activation=act)
    f, slope = block.activation(a, act)
    off = block.gated_grad_bounds(a, b, d_a, d_b, dh, act)
    within(dgate, dh.double() * b * slope, off[0], torch.bfloat16)
    within(dup, dh.double() * f, off[1], torch.bfloat16)
    within(gate.g, *sums(tokens, dgate.double().T, xv))
    within(up.g, *sums(tokens, dup.double().T, xv))
    B.pvt_mx_gated_grad_input(dgate, dup, ff.w_gate, ff.w_up, dn)
    both = torch.cat((dgate, dup), dim=1).double()
    within(dn, *sums(2 * INNER, both, torch.cat((gv, uv))), torch.bfloat16)
    want = block.norm_grad(total, stats, dn, kind, weight, dtotal)
    off = block.norm_grad_bounds(total, stats, dn, kind, weight, dtotal)
    within(dx, want[0], off[0], torch.bfloat16)
    within(ff.dweight, want[1], off[1])
    if bias is not None:
        within(ff.dbias, want[2], off[2])


def test_gradients_are_those_of_the_whole_by_differences():
    """Of the formulas in float64 from the held weights on, with the quantisation of activations taken for the identity: the direction
    of a small change of x changes the loss by its product with dx.  How far rounding to 4 bits moves dx is not asked; the formula's own
    dx is what the kernels' is compared with, stage by stage, above."""
    gen = torch.Generator("cuda").manual_seed(2)
    gv, uv, dv = (torch.randn(s, dtype=torch.float64, device="cuda", generator=gen) * 0.1 for s in ((24, 16), (24, 16), (16, 24)))
    weight = 1 + 0.2 * torch.randn(16, dtype=torch.float64, device="cuda", generator=gen)
    x, dy, dtotal, way = (torch.randn(5, 16, dtype=torch.float64, device="cuda", generator=gen) for _ in range(4))

    def loss(x):
        n = block.norm(x, block.RMS, 1e-5, weight)[0]
        return ((block.gated(n @ gv.T, n @ uv.T, block.SILU) @ dv.T) * dy).sum() + (x * dtotal).sum()

    n, mean, rstd = block.norm(x, block.RMS, 1e-5, weight)
    a, b = n @ gv.T, n @ uv.T
    f, slope = block.activation(a, block.SILU)
    dh = dy @ dv
    dn = (dh * b * slope) @ gv + (dh * f) @ uv
    dx = block.norm_grad(x, torch.cat((mean, rstd), dim=1), dn, block.RMS, weight, dtotal)[0]
    step = 1e-6
    assert abs((loss(x + step * way) - loss(x - step * way)).item() / (2 * step) - (dx * way).sum().item()) <= 1e-6 * (dx * way).abs().sum().item()


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
def test_steps_over_two_batches(fmt):
    """Gradients of two batches add up in the layers' g and the norm's, the V step and Adam take them, and the next pass has the weights
    that they leave."""
    gen = torch.Generator("cuda").manual_seed(7)
    gate, up, down = layers()
    weight, bias = torch.ones(WIDTH, device="cuda"), torch.zeros(WIDTH, device="cuda")
    ff = FeedForward(gate, up, down, weight, bias, kind=B.PVT_NORM_LAYER, fmt=fmt)
    batches = [[torch.randn(t, WIDTH, device="cuda", generator=gen).bfloat16() for _ in range(2)] for t in (60, 100)]
    seen = []
    for i, (x, dy) in enumerate(batches):
        y, total = ff.forward(x)
        assert total is x
        ff.backward(dy, first=True)
        seen.append([layer.g.clone() for layer in (gate, up, down)] + [ff.dweight.clone(), ff.dbias.clone()])
    for i, (x, dy) in enumerate(batches):
        ff.forward(x)
        ff.backward(dy, first=i == 0)
    for got, one, two in zip([gate.g, up.g, down.g, ff.dweight, ff.dbias], *seen):
        # added in binary32 (or 64) once more: half a step of the sum, and of what is added
        assert ((got.double() - one.double() - two.double()).abs() <= 2.0 ** -24 * (got.double().abs() + two.double().abs()) + 1e-30).all()
    before = [values(m) for m in (ff.w_gate, ff.w_up, ff.w_down)]
    for layer in (gate, up, down):
        g = layer.g.cpu().numpy()
        idx, _ = layer.step(300, W_hat=torch.empty(layer.rows, layer.cols, device="cuda"))
        assert layer.status() == 0
        assert np.array_equal(idx.cpu().numpy().astype(np.uint32), oracle.select(oracle.group_norms(g, layer.eta), 300))
    m, v = torch.zeros(WIDTH, device="cuda"), torch.zeros(WIDTH, device="cuda")
    moved = weight.clone()
    B.pvt_adam_update(weight, ff.dweight, m, v, step=1, lr=0.01)
    # a first step moves every weight by the rate, against its gradient
    assert torch.allclose(moved - weight, 0.01 * torch.sign(ff.dweight).float(), rtol=1e-3)
    ff.quantize()
    after = [values(m) for m in (ff.w_gate, ff.w_up, ff.w_down)]
    for layer, m, b4, now in zip((gate, up, down), (ff.w_gate, ff.w_up, ff.w_down), before, after):
        ts = None if m.tensor_scale is None else m.tensor_scale.item()
        assert torch.equal(now, mx.values(*mx.quantize(layer.dequant(), fmt, ts), fmt, ts)) and not torch.equal(now, b4)


def test_shapes_and_order_are_checked():
    gate, up, down = layers()
    ones = torch.ones(WIDTH, device="cuda")
    for bad in (lambda: FeedForward(gate, down, up, ones), lambda: FeedForward(gate, up, up, ones), lambda: FeedForward(gate, up, down, ones[:-1]),
                lambda: FeedForward(gate, up, down, ones, ones[:-1])):
        with pytest.raises(ValueError):
            bad()
    ff = FeedForward(gate, up, down, ones)
    with pytest.raises(RuntimeError):
        ff.backward(torch.zeros(3, WIDTH, device="cuda").bfloat16())
    with pytest.raises(ValueError):
        ff.forward(torch.zeros(3, WIDTH - 8, device="cuda").bfloat16())
