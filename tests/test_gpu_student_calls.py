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


@pytest.mark.parametrize("vocab", [1000, 1001, 1003])
def test_the_pass_over_a_vocabulary_of_any_size(vocab):
    """Logits in rows of a multiple of 8 elements serve as dy after the loss has written its gradient over them; rows of vocab
    elements do where that is a multiple of 8, and are refused otherwise before anything is written."""
    tokens, width, k = 40, 256, 30
    gen = torch.Generator("cuda").manual_seed(vocab)
    x, w = B.new_mx(tokens, width, B.PVT_MX_E8M0_32), B.new_mx(vocab, width, B.PVT_MX_E8M0_32)
    B.pvt_mx_quantize(x, torch.randn(tokens, width, device="cuda", generator=gen))
    B.pvt_mx_quantize(w, torch.randn(vocab, width, device="cuda", generator=gen) * 0.1)
    xv, wv = (ref.values(*ref.unpack(m.codes, m.scales, m.rows, width, m.format), m.format) for m in (x, w))
    teacher = torch.randn(tokens, vocab, device="cuda", generator=gen)
    idx, val = torch.empty(tokens, k, dtype=torch.int32, device="cuda"), torch.empty(tokens, k, device="cuda")
    B.pvt_distill_top(teacher, idx, val)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for pitch in ((vocab + 7) // 8 * 8, vocab):
        logits = torch.full((tokens, pitch), math.nan, dtype=torch.bfloat16, device="cuda")[:, :vocab]
        loss = torch.empty(tokens, device="cuda")
        dx, g = torch.full((tokens, width), 7.0, device="cuda"), torch.full((vocab, width), 7.0, device="cuda")
        B.pvt_mx_product(x, w, logits, status=status)
        B.pvt_distill_loss(B.make_distill(logits, idx, val), loss, grad=logits, status=status)
        if pitch % 8:
            with pytest.raises(B.PvtError):
                B.pvt_mx_grad_input(logits, w, dx, status=status)
            with pytest.raises(B.PvtError):
                B.pvt_mx_grad_weight(logits, x, g, status=status)
            assert (dx == 7).all() and (g == 7).all()
            continue
        B.pvt_mx_grad_input(logits, w, dx, status=status)
        B.pvt_mx_grad_weight(logits, x, g, status=status)
        dy = logits.double()
        # sums of n terms within n 2^-23 of the sum of magnitudes, and one rounding of the result
        assert ((dx.double() - dy @ wv).abs() <= (vocab + 4) * 2.0 ** -23 * (dy.abs() @ wv.abs())).all()
        assert ((g.double() - dy.T @ xv).abs() <= (tokens + 4) * 2.0 ** -23 * (dy.abs().T @ xv.abs())).all()
    assert status.item() == 0


def test_captured_steps_read_what_is_there_when_they_are_replayed():
    rows, vocab, k = 6, 9001, 40
    x, teacher = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, vocab, device="cuda")
    idx, val = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
    lse, weight = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    loss, stats, grad = torch.empty(rows, device="cuda"), torch.empty(rows, 8, device="cuda"), torch.empty_like(x)
    d = B.make_distill(x, idx, val, teacher_lse=lse, weight=weight)
    outs = (idx, val, lse, loss, stats, grad)

    def step():
        B.pvt_distill_top(teacher, idx, val, lse)
        B.pvt_distill_loss(d, loss, stats=stats)
        B.pvt_distill_grad(d, stats, grad)

    def fill(seed):
        gen = torch.Generator("cuda").manual_seed(seed)
        teacher.copy_(2.5 * torch.randn(rows, vocab, device="cuda", generator=gen))
        x.copy_(teacher + torch.randn(rows, vocab, device="cuda", generator=gen))
        weight.copy_(torch.rand(rows, device="cuda", generator=gen))

    fill(1)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    earlier = None
    for seed in (1, 2, 3):
        fill(seed)
        graph.replay()
        got = [o.clone() for o in outs]
        for o in outs:
            o.fill_(-7)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
        assert earlier is None or not torch.equal(earlier, got[3])
        earlier = got[3]


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k", [(700, 500, 20), (650, 2051, 128), (600, 3001, 200), (1200, 7, 5)])
def test_every_one_of_many_short_rows(rows, vocab, k, dtype, tail):
    """All rows, and every gradient beside its own probability."""
    temperature = 1.5  # (a binary32 number)
    gen = torch.Generator("cuda").manual_seed(vocab)
    teacher = 2.5 * torch.randn(rows, vocab, device="cuda", generator=gen)
    x = (0.9 * teacher + torch.randn(rows, vocab, device="cuda", generator=gen)).to(dtype)
    val, idx = torch.topk(teacher, k, dim=1)
    lse = torch.logsumexp(teacher.double() / temperature, dim=1).float() if tail else None
    loss, grad = torch.empty(rows, device="cuda"), torch.empty_like(x)
    B.pvt_distill_loss(B.make_distill(x, idx.int(), val.contiguous(), teacher_lse=lse, temperature=temperature), loss, grad=grad)
    logq = torch.log_softmax(x.double() / temperature, dim=1)
    logp = val.double() / temperature
    logp = logp - (torch.logsumexp(logp, dim=1) if lse is None else lse.double())[:, None]
    p = logp.exp()
    want = (p * (logp - torch.gather(logq, 1, idx))).sum(dim=1)
    target = torch.zeros_like(logq).scatter_(1, idx, p)
    if tail:
        rest = 1.0 - p.sum(dim=1)
        assert (rest > 1e-4).all()
        others = logq.scatter(1, idx, -math.inf)
        log_rest = torch.logsumexp(others, dim=1)
        want = want + rest * (rest.log() - log_rest)
        target = target + rest[:, None] * (others - log_rest[:, None]).exp()
    want_grad = (target.sum(dim=1, keepdim=True) * logq.exp() - target) / temperature
    # a probability is off by at most e of itself: 2^-22 of ex2, |log y| 2^-23 of the exponent (|log y| y sums to less than 20 of the
    # sum here) and n / 128 + 24 roundings of sums by 64 threads
    e = 2.0 ** -23 * (vocab / 128 + 40)
    assert ((loss.double() - want).abs() <= 2 * e + 2.0 ** -24 * want.abs()).all()
    eps, tiny = torch.finfo(dtype).eps / 2, torch.finfo(dtype).tiny
    bound = 2 * e * (logq.exp() + target) / temperature + eps * want_grad.abs() + tiny * eps + 1e-37
    assert ((grad.double() - want_grad).abs() <= bound).all()


def test_products_under_every_power_of_two():
    """All 255 scales of one operand beside a small, a middle and a large one of the other: exact wherever the result is well inside of
    binary32, and no result elsewhere disturbs its neighbours."""
    b = 32
    gen = torch.Generator("cuda").manual_seed(3)
    scales = [torch.arange(255, device="cuda")[:, None], torch.tensor([[20], [127], [235]], device="cuda")]
    ms, vs = [], []
    for s in scales:
        codes = torch.randint(0, 16, (s.shape[0], b), device="cuda", generator=gen)
        h, packed = ref.pack(codes, s, B.PVT_MX_E8M0_32)
        ms.append(B.make_mx(h, packed, s.shape[0], b, B.PVT_MX_E8M0_32))
        vs.append(ref.values(codes, s, B.PVT_MX_E8M0_32))
    y = torch.empty(3, 255, device="cuda")
    B.pvt_mx_product(ms[1], ms[0], y)
    want = vs[1] @ vs[0].T
    # (elements are multiples of 1/2 up to 6: sums of 32 products are multiples of 1/4 up to 1152, times the two scales)
    inside = (scales[0].T + scales[1] - 254).abs() <= 100
    assert inside.any(dim=0).all() and torch.equal(y[inside], want[inside].float())
    assert not torch.isnan(y[inside]).any()
    values = torch.empty(255, b, device="cuda")
    B.pvt_mx_dequant(ms[0], values)
    assert torch.equal(values, vs[0].float())
