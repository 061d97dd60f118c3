"""The calls of a training step one after the other, as they are used: quantised weights and activations, their product, the loss
against a teacher's list, its gradient, the gradient of the weights into the layer's g, and the V step on it."""
import numpy as np
import pytest
import torch

import student_reference as ref
from oracle import pvt_oracle as oracle
from paper_2405_14852_b200 import binding as B
from paper_2405_14852_b200 import synth
from paper_2405_14852_b200.vstep import VStepLayer

pytestmark = pytest.mark.gpu


def step(dev, x, teacher, fmt, k, tail, batches, graph=False):
    """One step over `batches` slices of the tokens; returns losses and what was held."""
    tokens, vocab = teacher.shape
    w = dev.quantized(fmt)
    idx = torch.empty(tokens, k, dtype=torch.int32, device="cuda")
    val, lse = torch.empty(tokens, k, device="cuda"), torch.empty(tokens, device="cuda")
    loss = torch.empty(tokens, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    logits = torch.empty(tokens, vocab, dtype=torch.bfloat16, device="cuda")
    dx = torch.empty(tokens, x.shape[1], device="cuda")
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    per = tokens // batches
    held = [B.new_mx(per, x.shape[1], fmt) for _ in range(batches)]

    def run():
        B.pvt_distill_top(teacher, idx, val, lse)
        for i, m in enumerate(held):
            at = slice(i * per, (i + 1) * per)
            B.pvt_mx_quantize(m, x[at])
            B.pvt_mx_product(m, w, logits[at], status=status)
            d = B.make_distill(logits[at], idx[at], val[at], teacher_lse=lse[at] if tail else None, weight=weight[at])
            B.pvt_distill_loss(d, loss[at], grad=logits[at], status=status)  # the gradient takes the logits' place
            B.pvt_mx_grad_input(logits[at], w, dx[at], status=status)
            dev.accumulate_grad(logits[at], m, first=i == 0)

    run()
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        for t in (loss, dx, dev.g):
            t.fill_(7.0)
        g.replay()
    torch.cuda.synchronize()
    assert status.item() == 0
    return loss, dx, w, held, idx, val, lse, logits


@pytest.mark.parametrize("fmt", [B.PVT_MX_E8M0_32, B.PVT_MX_E4M3_16])
@pytest.mark.parametrize("tokens,batches,tail,graph", [(6, 1, False, False), (64, 2, True, False), (320, 2, False, True)])
def test_a_training_step_down_to_the_chosen_groups(fmt, tokens, batches, tail, graph):
    vocab, width, k = 1000, 256, 40  # the layer is the model's last: vocab x width
    L = synth.make_layer(vocab, width, cfg=71, codebook_size=256, codebook_fp16=True)
    dev = VStepLayer.from_host(L)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn(tokens, width, device="cuda", generator=gen).bfloat16()
    teacher = (x.float() @ dev.W.T * 4).bfloat16()
    loss, dx, w, held, idx, val, lse, dlogits = step(dev, x, teacher, fmt, k, tail, batches, graph)

    # the list, from its definition
    want_idx, want_val, _ = ref.top(teacher, k)
    assert torch.equal(idx.long(), want_idx) and torch.equal(val.double(), want_val)
    # every later call from what it was given: values of the held matrices, logits rounded to bfloat16
    wv = ref.values(*ref.unpack(w.codes, w.scales, vocab, width, fmt), fmt)
    per = tokens // batches
    xv = torch.cat([ref.values(*ref.unpack(m.codes, m.scales, per, width, fmt), fmt) for m in held])
    exact = xv @ wv.T
    # bfloat16 logits: within half a step of the sum, which is within (width + 4) 2^-23 of the sum of magnitudes
    slack = 2.0 ** -8 * exact.abs() + (width + 4) * 2.0 ** -23 * (xv.abs() @ wv.abs().T)
    want_loss, want_grad = ref.distill(exact, idx, val, lse if tail else None, torch.full((tokens,), 1.0 / tokens))
    # logits off by `slack` move the loss by at most twice the largest of them, a probability by as much of itself
    worst = slack.amax(dim=1).cpu()
    assert ((loss.cpu().double() - want_loss).abs() * tokens <= 2 * worst + 1e-4).all()
    bound = (4 * worst[:, None] + 2.0 ** -8) * (want_grad.abs() + torch.softmax(exact, dim=1).cpu() / tokens) + 1e-7 / tokens
    assert ((dlogits.cpu().double() - want_grad).abs() <= bound).all()
    # gradients of weights and inputs, exactly from the bfloat16 gradient that was there
    dy = dlogits.double()
    want_g = dy.T @ xv
    assert ((dev.g.double() - want_g).abs() <= (tokens + 4) * 2.0 ** -23 * (dy.abs().T @ xv.abs())).all()
    assert ((dx.double() - dy @ wv).abs() <= (vocab + 4) * 2.0 ** -23 * (dy.abs() @ wv.abs())).all()

    # and the V step takes it
    chosen = 200
    got, _ = dev.step(chosen, W_hat=torch.empty(vocab, width, device="cuda"))
    torch.cuda.synchronize()
    assert dev.status() == 0
    g = dev.g.cpu().numpy()
    assert np.array_equal(got.cpu().numpy().astype(np.uint32), oracle.select(oracle.group_norms(g, L.eta), chosen))


def test_tensors_of_another_device_or_shape_are_refused():
    x = torch.randn(4, 64, device="cuda")
    m = B.new_mx(4, 64, B.PVT_MX_E8M0_32)
    for bad in (lambda: B.pvt_mx_quantize(m, x.cpu()), lambda: B.pvt_mx_quantize(m, x[:3]), lambda: B.pvt_mx_quantize(m, x.double()),
                lambda: B.pvt_mx_quantize(m, torch.randn(64, 4, device="cuda").T), lambda: B.pvt_mx_quantize(m, x[:1].expand(4, 64)),
                lambda: B.pvt_mx_product(m, m, torch.empty(4, 5, device="cuda")),
                lambda: B.pvt_mx_grad_input(x, m, torch.empty(4, 64, device="cuda")),
                lambda: B.pvt_mx_grad_weight(torch.zeros(4, 8, device="cuda").bfloat16(), m, torch.empty(8, 64, device="cuda").half()),
                lambda: B.pvt_distill_top(x, torch.empty(4, 3, device="cuda"), torch.empty(4, 3, device="cuda")),
                lambda: B.make_mx(m.codes, m.scales.cpu(), 4, 64, B.PVT_MX_E8M0_32)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.PvtError):
        B.pvt_mx_grad_input(torch.zeros(4, 20, device="cuda").bfloat16(), B.new_mx(20, 64, 0), torch.empty(4, 64, device="cuda"))
