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
