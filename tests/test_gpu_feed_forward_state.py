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
