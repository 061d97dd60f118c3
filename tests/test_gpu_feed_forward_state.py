"""The feed-forward half of a block over its lifetime: layers of zeros, weights that change under a captured pass, what is kept between
forward and backward, scales of activations, gradients' types, waits that run out."""
import warnings

import pytest
import torch

import block_reference as block
from paper_2405_14852_b200 import binding as B
from paper_2405_14852_b200.vstep import FeedForward
from test_gpu_feed_forward import INNER, WIDTH, layers, sums, values, within

pytestmark = pytest.mark.gpu


def ones():
    return torch.ones(WIDTH, device="cuda")


def batch(seed, tokens=50, n=1):
    gen = torch.Generator("cuda").manual_seed(seed)
    made = [torch.randn(tokens, WIDTH, device="cuda", generator=gen).bfloat16() for _ in range(n)]
    return made[0] if n == 1 else made


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("zeros", [("down",), ("gate", "up"), ("gate",)])
def test_layers_of_zeros(fmt, zeros):
    """A layer that starts at 0 gives 0, and the gradient that takes it away from there."""
    gate, up, down = layers()
    for name in zeros:
        dict(gate=gate, up=up, down=down)[name].scale.zero_()
    ff = FeedForward(gate, up, down, ones(), fmt=fmt)
    x, dy = batch(1, n=2)
    y, _ = ff.forward(x)
    dx = ff.backward(dy, first=True)
    assert not y.any()
    for t in (dx, gate.g, up.g, down.g, ff.dweight):
        assert torch.isfinite(t).all()
    if zeros == ("down",):
        hv = values(ff._kept[3])
        within(down.g, *sums(50, dy.double().T, hv))
        assert down.g.any()


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
def test_captured_passes_read_the_weights_of_the_last_quantisation(fmt):
    made = layers()
    ff = FeedForward(*made, ones(), fmt=fmt)
    x, dy = batch(2, n=2)
    ff.forward(x), ff.backward(dy, first=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = ff.forward(x)
        dx = ff.backward(dy, first=True)
    for factor in (3.0, 0.01):
        for layer in made:
            layer.scale.mul_(factor)
        ff.quantize()
        filler = [torch.full((1,), 5.0, device="cuda") for _ in range(64)]  # (what a scale of its own would have left free)
        graph.replay()
        got = [t.clone() for t in (y, dx, *(layer.g for layer in made), ff.dweight)]
        fresh = FeedForward(*made, ones(), fmt=fmt)
        want = [fresh.forward(x)[0], fresh.backward(dy, first=True), *(layer.g for layer in made), fresh.dweight]
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(filler) == 64


def held_within(m, want, slack, ts):
    """The values of a 4-bit matrix under e4m3 scales are near the numbers that were quantised, which are `want` to within `slack`.

    With a the largest magnitude of a block, d = scale * ts its unit: the scale is rounded to 3 bits, by a sixteenth of it and by 2^-10 where
    it is below 2^-6, so 6 d is between 15/16 a - 6 ts 2^-10 and 17/16 a + 6 ts 2^-10.  Elements are 0, 0.5, 1, 1.5, 2, 3, 4, 6 units:
    a number below 2 d moves by d / 4 at most, one between 2 d and 6 d by a fifth of itself, one beyond 6 d down to it."""
    n = m.cols // 16 * 16
    top = (want.abs() + slack)[:, :n].view(m.rows, -1, 16).amax(dim=2).repeat_interleave(16, dim=1)
    d = top * (17 / 96) + ts * 2.0 ** -10
    bound = torch.maximum(torch.maximum(0.2 * (want[:, :n].abs() + slack[:, :n]), d / 4), top / 16 + 6 * ts * 2.0 ** -10)
    off = (values(m)[:, :n] - want[:, :n]).abs()
    assert (off <= 1.0001 * (bound + slack[:, :n])).all()


@pytest.mark.parametrize("std", [0.00625, 0.05, 20.0])
@pytest.mark.parametrize("kind,act", [(B.PVT_NORM_RMS, B.PVT_ACT_SILU), (B.PVT_NORM_LAYER, B.PVT_ACT_GELU)])
def test_activations_of_any_size_under_e4m3(std, kind, act):
    """a and b of a deviation of 0.1, 0.8 and 320, so h of 0.005, 0.3 and 50 000: neither lost below the smallest scale nor cut off beyond
    the largest one."""
    made = layers(std)
    weight = ones() * 0.01  # (n is small as well)
    for layer in made[:2]:
        layer.scale.mul_(100.0)
    ff = FeedForward(*made, weight, kind=kind, activation=act, fmt=B.PVT_MX_E4M3_16)
    (x, residual), (first, r1) = batch(3, 300, 2), batch(4, 200, 2)
    ff.take_scales(first, r1)
    kept = ff.x_scale, ff.h_scale
    ff.take_scales(x, residual, room=1.0)
    assert ff.x_scale is kept[0] and ff.h_scale is kept[1]
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        y, total = ff.forward(x, residual)
    _, _, xq, hq = ff._kept
    held_within(xq, block.norm(total, kind, 1e-5, weight)[0], block.norm_bounds(total, kind, 1e-5, weight)[0], ff.x_scale.double())
    a, b, d_a, d_b = block.products(values(xq), values(ff.w_gate), values(ff.w_up))
    h = block.gated(a, b, act)
    held_within(hq, h, block.gated_bound(a, b, d_a, d_b, act), ff.h_scale.double())
    # the largest one is there: room 1 is this batch's own
    assert values(hq).abs().max() >= 0.8 * h.abs().max() and values(xq).any(dim=1).all()
    dy = batch(5, 300)
    ff.backward(dy, first=True)
    within(made[2].g, *sums(300, dy.double().T, values(hq)))
    again = FeedForward(*made, weight, kind=kind, activation=act, fmt=B.PVT_MX_E4M3_16, x_scale=kept[0], h_scale=kept[1])
    assert torch.equal(again.forward(x, residual)[0], y)


def test_scales_of_activations_are_checked():
    made = layers()
    one = torch.ones(1, device="cuda")
    for bad in (dict(x_scale=one), dict(fmt=B.PVT_MX_E4M3_16, h_scale=one.half()), dict(fmt=B.PVT_MX_E4M3_16, x_scale=one.expand(2))):
        with pytest.raises(ValueError):
            FeedForward(*made, ones(), **bad)
    x = batch(6)
    with pytest.raises(ValueError):
        FeedForward(*made, ones()).take_scales(x)
    with pytest.raises(ValueError):
        FeedForward(*made, ones(), fmt=B.PVT_MX_E4M3_16, x_scale=torch.ones(1), h_scale=one).forward(x)
    ff = FeedForward(*made, ones(), fmt=B.PVT_MX_E4M3_16, x_scale=one)
    with pytest.warns(UserWarning, match="h_scale"):
        ff.forward(x)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        ff.forward(x)
        FeedForward(*made, ones()).forward(x)


@pytest.mark.parametrize("tokens", [3, 200])
@pytest.mark.parametrize("name", ["pvt_mx_gated", "pvt_mx_product", "pvt_mx_grad_input", "pvt_mx_grad_weight", "pvt_mx_gated_grad",
                                  "pvt_mx_gated_grad_input"])
def test_a_wait_that_runs_out_in_any_call_is_reported(name, tokens, monkeypatch):
    """One call of a pass has the bound of its on-chip waits lowered and leaves out a copy; see the test of the search kernels' waits."""
    made = layers()
    ff = FeedForward(*made, ones())
    x, dy = batch(7, tokens, 2)

    def a_pass():
        y, _ = ff.forward(x)
        return [y, ff.backward(dy, first=True), *(layer.g.clone() for layer in made), ff.dweight.clone()]

    want = a_pass()
    assert ff.status() == 0
    call = getattr(B, name)

    def held_up(*args, **kw):
        torch.cuda.synchronize()
        B.pvt_test_wait_limit(20000, 0)
        try:
            call(*args, **kw)
            torch.cuda.synchronize()
        finally:
            B.pvt_test_wait_limit(0, -1)

    with monkeypatch.context() as m:
        m.setattr(B, name, held_up)
        a_pass()
    assert ff.status() & B.PVT_DEV_WAIT_EXPIRED and ff.status() == 0
    assert all(torch.equal(a, b) for a, b in zip(a_pass(), want)) and ff.status() == 0


@pytest.mark.parametrize("with_residual", [False, True])
def test_what_is_kept_for_backward_may_not_be_written_to(with_residual):
    """The residual stream carried on in place, as x += y does, is another row of numbers than the one that was normalised."""
    ff = FeedForward(*layers(), ones())
    x, residual, dy = batch(8, n=3)
    args = (x, residual) if with_residual else (x,)
    ff.forward(*args)
    want = ff.backward(dy, first=True)
    for write in (lambda total, y: total.add_(y), lambda total, y: total[3:5].zero_(), lambda total, y: total.view(-1).mul_(1)):
        y, total = ff.forward(*args)
        keep = total.clone()
        write(total, y)
        with pytest.raises(RuntimeError):
            ff.backward(dy, first=True)
        total.copy_(keep)
        y, total = ff.forward(*args)
        assert torch.equal(ff.backward(dy, first=True), want)
        total.add_(y)  # (behind backward it may)
        total.copy_(keep)
    with torch.inference_mode():
        y, total = ff.forward(*(t.clone() for t in args))
        assert torch.equal(ff.backward(dy, first=True), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens", [5, 300])
def test_gradients_of_the_residual_stream_in_its_own_type(dtype, tokens):
    """dx is as near to its formula as its type allows: nothing on the way from dgate and dup is rounded to fewer bits."""
    gen = torch.Generator("cuda").manual_seed(tokens)
    made = layers()
    ff = FeedForward(*made, 1 + 0.2 * torch.randn(WIDTH, device="cuda", generator=gen), grad_dtype=dtype)
    x, residual, dtotal = (torch.randn(tokens, WIDTH, device="cuda", generator=gen).to(dtype) for _ in range(3))
    dy = batch(9, tokens)
    _, total = ff.forward(x, residual)
    dx = ff.backward(dy, dtotal, first=True)
    assert dx.dtype == dtype and total.dtype == dtype
    _, stats, xq, _ = ff._kept
    dh, dgate, dup = (torch.empty(tokens, INNER, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    B.pvt_mx_grad_input(dy, ff.w_down, dh)
    B.pvt_mx_gated_grad(xq, ff.w_gate, ff.w_up, dh, dgate, dup)
    dn, off = sums(2 * INNER, torch.cat((dgate, dup), dim=1).double(), torch.cat((values(ff.w_gate), values(ff.w_up))))
    off = off + block.rounding(dn.abs() + off, dtype)
    want = block.norm_grad(total, stats, dn, block.RMS, ff.weight, dtotal)[0]
    # the norm's gradient is linear in dn: what moves an element of dn by `off` moves dx by no more than with all signs alike
    xh, rstd, w = (total.double() - stats[:, :1].double()) * stats[:, 1:].double(), stats[:, 1:].double(), ff.weight.double().abs()
    moved = rstd * (w * off + xh.abs() * (w * off * xh.abs()).mean(dim=1, keepdim=True))
    within(dx, want, moved + block.norm_grad_bounds(total, stats, dn, block.RMS, ff.weight, dtotal)[0], dtype)


def test_types_of_gradients_are_checked():
    made = layers()
    with pytest.raises(ValueError):
        FeedForward(*made, ones(), grad_dtype=torch.float64)
    ff = FeedForward(*made, ones())
    x, dy = batch(10, n=2)
    ff.forward(x)
    before = made[2].g.clone()
    for dtotal in (dy.float(), dy[:-1], dy.T.contiguous().T):
        with pytest.raises(ValueError):
            ff.backward(dy, dtotal, first=True)
    assert torch.equal(made[2].g, before)  # nothing has been started


def test_captured_passes_keep_their_workspace_when_larger_batches_follow():
    """What a captured backward pass writes to stays its own: nothing that is allocated afterwards is written to by its replays."""
    ff = FeedForward(*layers(), ones())
    x, dy = batch(11, 5, 2)
    ff.forward(x), ff.backward(dy, first=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ff.forward(x)
        dx = ff.backward(dy, first=True)
    graph.replay()
    want = dx.clone(), ff.dweight.clone()
    small = B.pvt_norm_workspace_bytes(B.make_norm(x))
    big, dbig = batch(12, 3001, 2)
    ff.forward(big), ff.backward(dbig, first=True)
    # (takes every block of that size that is free)
    filler = [torch.full((small,), 0x5a, dtype=torch.uint8, device="cuda") for _ in range(256)]
    graph.replay()
    assert torch.equal(dx, want[0]) and torch.equal(ff.dweight, want[1])
    assert all((t == 0x5a).all() for t in filler)
