"""The feed-forward half of a block over its lifetime: layers of zeros, weights that change under a captured pass, what is kept between
forward and backward, scales of activations, gradients' types, waits that run out."""
import pytest
import torch

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
