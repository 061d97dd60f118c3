"""Calls on the pass that g comes from as a user may make them: one row of a wider matrix, matrices given to be written, logits of a
vocabulary of any size, steps replayed on other data, every scale."""
import math
import warnings

import pytest
import torch

import student_reference as ref
from paper_2405_14852_b200 import binding as B
from paper_2405_14852_b200 import synth
from paper_2405_14852_b200.vstep import VStepLayer

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", TYPES)
def test_one_row_in_place_however_far_the_next_would_be(dtype):
    """The distance of rows says nothing where there is one: two views of it may differ there."""
    wide = torch.randn(3, 1040, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
    logits = wide[1:2, :1000]
    same = wide[1, :1000].view(1, 1000)
    assert logits.data_ptr() == same.data_ptr() and logits.stride(0) != same.stride(0)
    idx = torch.arange(7, dtype=torch.int32, device="cuda")[None]
    val = torch.randn(1, 7, device="cuda")
    keep, others = logits.clone(), wide.clone()
    loss, want, stats = torch.empty(1, device="cuda"), torch.empty(1, 1000, dtype=dtype, device="cuda"), torch.empty(1, 8, device="cuda")
    d = B.make_distill(logits, idx, val)
    B.pvt_distill_loss(d, loss, grad=want, stats=stats)
    B.pvt_distill_loss(d, loss, grad=same)
    assert torch.equal(logits, want)
    logits.copy_(keep)
    B.pvt_distill_grad(d, stats, same)
    assert torch.equal(logits, want)
    logits.copy_(keep)
    assert torch.equal(wide, others)  # nothing beside the row was written


def test_weights_into_a_given_matrix():
    """Its format and scale count; another format or scale beside it is refused, not passed over."""
    dev = VStepLayer.from_host(synth.make_layer(64, 256, cfg=71, codebook_size=256, codebook_fp16=True))
    scale, other = torch.tensor([0.01], device="cuda"), torch.tensor([0.02], device="cuda")
    fine = B.new_mx(64, 256, B.PVT_MX_E4M3_16, tensor_scale=scale)
    coarse, plain = B.new_mx(64, 256, B.PVT_MX_E8M0_32), B.new_mx(64, 256, B.PVT_MX_E4M3_16)
    for m, alike in ((fine, [dict(), dict(fmt=B.PVT_MX_E4M3_16), dict(tensor_scale=scale), dict(fmt=B.PVT_MX_E4M3_16, tensor_scale=scale)]),
                     (coarse, [dict(), dict(fmt=B.PVT_MX_E8M0_32)]), (plain, [dict(), dict(fmt=B.PVT_MX_E4M3_16)])):
        want = dev.quantized(m.format, m.tensor_scale)
        for kw in alike:
            m.codes.fill_(0xa5)
            assert dev.quantized(out=m, **kw) is m
            assert torch.equal(m.codes, want.codes) and torch.equal(m.scales, want.scales)
    assert dev.quantized().format == B.PVT_MX_E8M0_32
    before = fine.codes.clone()
    for m, kw in ((fine, dict(fmt=B.PVT_MX_E8M0_32)), (coarse, dict(fmt=B.PVT_MX_E4M3_16)), (fine, dict(tensor_scale=other)),
                  (plain, dict(tensor_scale=scale)), (coarse, dict(tensor_scale=scale))):
        with pytest.raises(ValueError):
            dev.quantized(out=m, **kw)
    assert torch.equal(fine.codes, before)


def test_small_weights_under_e4m3_scales_are_warned_of_and_kept_with_a_tensor_scale():
    """Without a factor for the matrix the scales of small blocks are 0.  With the one that the documentation names an element is off by
    no more than its rounding and its block's scale's."""
    dev = VStepLayer.from_host(synth.make_layer(256, 512, cfg=71, codebook_size=256, codebook_fp16=True))
    dev.scale.mul_(0.001 / dev.dequant().std())
    w_hat = dev.dequant()
    with pytest.warns(UserWarning, match="tensor_scale"):
        lost = dev.quantized(B.PVT_MX_E4M3_16)
    with pytest.warns(UserWarning, match="tensor_scale"):
        dev.quantized(out=lost)
    values = torch.empty_like(w_hat)
    B.pvt_mx_dequant(lost, values)
    assert (values == 0).float().mean() > 0.5
    scale = (w_hat.abs().amax() / (6 * 448)).reshape(1)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        kept = dev.quantized(B.PVT_MX_E4M3_16, tensor_scale=scale)
        dev.quantized(out=kept)
        dev.quantized()
    B.pvt_mx_dequant(kept, values)
    block = w_hat.view(256, -1, 16).abs().amax(dim=2).repeat_interleave(16, dim=1)
    # half of the widest step between elements, 2 of 6, and the scale's own rounding, 2^-4, of the largest; its smallest is 2^-9
    assert ((values - w_hat).abs() <= block * (1 / 6 + 1 / 16) + 6 * 2.0 ** -10 * scale).all()
