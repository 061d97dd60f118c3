"""Calls on the pass that g comes from as a user may make them: one row of a wider matrix, matrices given to be written, logits of a
vocabulary of any size, steps replayed on other data, every scale."""
import math

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
