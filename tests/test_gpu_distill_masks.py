"""Distillation where masks, far logits or a complete list leave sums that are nothing or nearly nothing, against float64."""
import math

import pytest
import torch

from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def exact(x, idx, val, lse, temperature):
    """Loss, gradient, q and (for bounds) each row's p and unlisted target of whole tensors in float64; every entry is listed once."""
    logq = torch.log_softmax(x.double() / temperature, dim=1)
    at = idx.long()
    logp = val.double() / temperature
    logp = logp - (torch.logsumexp(logp, dim=1) if lse is None else lse.double())[:, None]
    p = logp.exp()
    loss = torch.where(p > 0, p * (logp - torch.gather(logq, 1, at)), 0.0).sum(dim=1)
    listed = torch.zeros_like(logq).scatter_(1, at, p)
    unlisted = torch.zeros_like(logq)
    if lse is not None:
        rest = (1.0 - p.sum(dim=1)).clamp(min=0.0)
        others = logq.scatter(1, at, -math.inf)
        log_rest = torch.logsumexp(others, dim=1)
        loss = loss + torch.where(rest > 0, rest * (rest.log() - log_rest), 0.0)
        share = (others - log_rest[:, None]).exp()
        unlisted = torch.where(torch.isfinite(log_rest)[:, None], rest[:, None] * share, 0.0)
    whole = listed.sum(dim=1) + (0.0 if lse is None else rest)
    q = logq.exp()
    return loss, (whole[:, None] * q - listed - unlisted) / temperature, q, listed, unlisted


def calls(x, idx, val, lse, temperature):
    """Loss and gradient by one call, by two and in place: all the same."""
    d = B.make_distill(x, idx, val, teacher_lse=lse, temperature=temperature)
    rows = x.shape[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, grad = torch.full((rows,), math.nan, device="cuda"), torch.full_like(x, math.nan, memory_format=torch.contiguous_format)
    B.pvt_distill_loss(d, loss, grad=grad, status=status)
    again, stats, grad2 = torch.empty_like(loss), torch.empty(rows, B.PVT_DISTILL_STATS, device="cuda"), torch.empty_like(grad)
    B.pvt_distill_loss(d, again, stats=stats, status=status)
    B.pvt_distill_grad(d, stats, grad2, status=status)
    same = lambda a, b: bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())  # noqa: E731
    assert same(loss, again) and same(grad, grad2)
    copy = x.clone()
    B.pvt_distill_loss(B.make_distill(copy, idx, val, teacher_lse=lse, temperature=temperature), again, grad=copy, status=status)
    assert same(loss, again) and same(grad, copy)
    assert status.item() == 0
    return loss, grad


def off(vocab):
    """What a probability may be off by, of itself: 2^-22 of ex2, |log y| 2^-23 of the exponent (|log y| y sums to less than 20 of
    the sum here) and n / 512 + 24 roundings of sums."""
    return 2.0 ** -23 * (vocab / 1024 + 40)


def near(loss, grad, want, vocab, temperature=1.0):
    want_loss, want_grad, q, listed, unlisted = want
    e = off(vocab)
    assert ((loss.double() - want_loss).abs() <= 2 * e + 2.0 ** -24 * want_loss.abs()).all()
    eps, tiny = torch.finfo(grad.dtype).eps / 2, torch.finfo(grad.dtype).tiny
    bound = (2 * e * (q + unlisted) + 2.0 ** -23 * listed) / temperature + eps * want_grad.abs() + tiny * eps + 1e-37
    assert ((grad.double() - want_grad).abs() <= bound).all()


# rows and vocabulary: a block to a row, few threads to a row, several blocks to a row
FORMS = [(3, 1000), (700, 1000), (2, 66000)]


def masked_beyond_the_list(rows, vocab, k, mask, order):
    """20 entries allowed; the teacher has `mask` elsewhere, the student -infinity; the list holds them and masked entries."""
    gen = torch.Generator("cuda").manual_seed(k)
    keep = torch.randperm(vocab, device="cuda", generator=gen)[:k]
    x = torch.full((rows, vocab), -math.inf, device="cuda")
    x[:, keep[:20]] = torch.randn(rows, 20, device="cuda", generator=gen)
    val = torch.full((rows, k), mask, device="cuda")
    val[:, :20] = 2.0 * torch.randn(rows, 20, device="cuda", generator=gen)
    idx = keep.int().expand(rows, k).contiguous()
    if order != "first":
        at = torch.arange(k - 1, -1, -1, device="cuda") if order == "last" else torch.randperm(k, device="cuda", generator=gen)
        idx, val = idx[:, at].contiguous(), val[:, at].contiguous()
    return x, idx, val


@pytest.mark.parametrize("order", ["first", "last", "mixed"])
@pytest.mark.parametrize("mask", [-1e4, -65504.0, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("k", [20, 32, 33, 64, 300])
@pytest.mark.parametrize("rows,vocab", FORMS)
def test_listed_entries_that_the_teacher_masks_with_a_number_and_the_student_with_infinity(rows, vocab, k, mask, order):
    """Their probability is 0 in any precision, so they add nothing, whichever threads look at them."""
    x, idx, val = masked_beyond_the_list(rows, vocab, k, mask, order)
    loss, grad = calls(x, idx, val, None, 1.0)
    assert torch.isfinite(loss).all()
    near(loss, grad, exact(x, idx, val, None, 1.0), vocab)


@pytest.mark.parametrize("rows,vocab", FORMS)
def test_probabilities_that_vanish_in_binary64_from_the_largest_listed_logit(rows, vocab):
    """exp(-700) is a number, exp(-800) is not, although exp(-100) of it would be: the student may have no mass there."""
    x, idx, val = masked_beyond_the_list(rows, vocab, 300, -800.0, "first")
    val[:, 20:] -= 10 * torch.rand(rows, 280, device="cuda")
    val[:, 100] = -700.0
    x[:, idx[0, 100]] = 0.5
    loss, grad = calls(x, idx, val, None, 1.0)
    near(loss, grad, exact(x, idx, val, None, 1.0), vocab)


def test_the_largest_listed_logit_is_that_of_an_entry_which_counts():
    """A repeated entry and one outside the vocabulary are left out: their logits, far above all others, are too."""
    x, idx, val = masked_beyond_the_list(1, 1000, 300, -1e4, "first")
    want = exact(x, idx, val, None, 1.0)
    wrong = torch.cat([torch.tensor([[1000, 2 ** 30]], dtype=torch.int32, device="cuda"), idx, idx[:, :3]], dim=1).contiguous()
    high = torch.cat([torch.full((1, 2), 3e4, device="cuda"), val, torch.full((1, 3), 2e4, device="cuda")], dim=1).contiguous()
    loss, grad = torch.empty(1, device="cuda"), torch.empty(1, 1000, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pvt_distill_loss(B.make_distill(x, wrong, high), loss, grad=grad, status=status)
    assert status.item() == B.PVT_DEV_BAD_INDEX
    near(loss, grad, want, 1000)
