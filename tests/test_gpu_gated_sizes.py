"""Gated products at the ends of the range of sizes."""
import pytest
import torch

import student_reference as mx
from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_outputs_beyond_30_bits():
    """Few tokens by more than 2^30 outputs into 4 bits (33 GB): no block writes to another's columns.  All weights are 0 but those of 300
    outputs from 2^30 - 100 on, whose codes are 1 (0x22) or 0.5 (0x11); x is 1.  Every product is a small number of binary32."""
    n, first, some = 2 ** 30 + 2 ** 20, 2 ** 30 - 100, 300
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 45e9:
        pytest.skip("needs 45 GB")
    codes = torch.zeros(n, 16, dtype=torch.uint8, device="cuda")
    codes[first:first + some] = 0x22
    codes[first:first + some:3] = 0x11
    scales = torch.full((B.pvt_mx_scale_bytes(n, 32, B.PVT_MX_E8M0_32),), 127, dtype=torch.uint8, device="cuda")
    w = B.make_mx(codes, scales, n, 32, B.PVT_MX_E8M0_32)
    x = B.new_mx(2, 32, B.PVT_MX_E8M0_32)
    B.pvt_mx_quantize(x, torch.ones(2, 32, device="cuda"))
    out = B.new_mx(2, n, B.PVT_MX_E8M0_32)
    out.codes.fill_(0xa5), out.scales.fill_(0xa5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pvt_mx_gated(x, w, w, quantized=out, status=status)
    # a = b = 32 or 16, and silu(a) = a to 2^-23: h is 1024 or 256
    h = torch.zeros(2, 1024, device="cuda")
    at = first % 256
    h[:, at:at + some] = 1024.0
    h[:, at:at + some:3] = 256.0
    want, want_scales = mx.pack(*mx.quantize(h, B.PVT_MX_E8M0_32), B.PVT_MX_E8M0_32)
    start = (first - at) // 2
    assert torch.equal(out.codes[:, start:start + 512], want)
    assert not out.codes[:, :start].any() and not out.codes[:, start + 512:n // 2].any()
    tiles = (first - at) // 128 * 512
    assert torch.equal(out.scales[tiles:tiles + want_scales.numel()], want_scales)
    assert not out.scales[:tiles].any() and not out.scales[tiles + want_scales.numel():].any() and status.item() == 0
