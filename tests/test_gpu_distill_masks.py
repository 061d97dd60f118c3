"""Distillation where masks, far logits or a complete list leave sums that are nothing or nearly nothing, against float64."""
import math

import pytest
import torch

from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def exact(x, idx, val, lse, temperature, rest=True):
    """Loss, gradient, q and (for bounds) each row's p and unlisted target of whole tensors in float64; every entry is listed once.
    With rest=False the teacher's remaining mass is 0 whatever its lse says."""
    temperature = torch.tensor(temperature).item()  # (the binary32 number that the call takes: 1.5e-8 off at 0.1)
    logq = torch.log_softmax(x.double() / temperature, dim=1)
    at = idx.long()
    logp = val.double() / temperature
    logp = logp - (torch.logsumexp(logp, dim=1) if lse is None else lse.double())[:, None]
    p = logp.exp()
    loss = torch.where(p > 0, p * (logp - torch.gather(logq, 1, at)), 0.0).sum(dim=1)
    listed = torch.zeros_like(logq).scatter_(1, at, p)
    unlisted = torch.zeros_like(logq)
    if lse is not None:
        rest = (1.0 - p.sum(dim=1)).clamp(min=0.0) * rest
        others = logq.scatter(1, at, -math.inf)
        log_rest = torch.logsumexp(others, dim=1)
        loss = loss + torch.where(rest > 0, rest * (rest.log() - log_rest), 0.0)
        # (relative to the largest of them: beside -3.4e38 the logarithm of a sum is not representable, its terms' shares are)
        share = torch.softmax((x.double() / temperature).scatter(1, at, -math.inf), dim=1)
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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,temperature", [(50.0, 1.0), (100.0, 1.0), (1e3, 1.0), (1e4, 1.0), (2e4, 3.0), (20.0, 0.1), (300.0, 0.1)])
@pytest.mark.parametrize("rows,vocab,k", [(3, 1000, 40), (700, 1000, 40), (2, 66000, 300)])
def test_unlisted_logits_far_below_the_listed_ones(rows, vocab, k, gap, temperature, dtype):
    """The rest of the student's mass is no binary32 number beside the listed, but it is a number: so are the loss, a
    multiple of its logarithm, and the gradient, which hands the rest of the teacher's mass to the unlisted by their shares of it."""
    gen = torch.Generator("cuda").manual_seed(k)
    keep = torch.stack([torch.randperm(vocab, device="cuda", generator=gen)[:k] for _ in range(rows)])
    x = torch.randn(rows, vocab, device="cuda", generator=gen) * min(temperature, 1.0) - gap
    x[0, ::3] = -math.inf
    x[1, : vocab // 2] = -gap * 2
    x.scatter_(1, keep, torch.randn(rows, k, device="cuda", generator=gen))
    x = x.to(dtype)
    val = torch.randn(rows, k, device="cuda", generator=gen) * temperature
    lse = torch.logsumexp(val.double() / temperature, dim=1).float() + 0.2  # the list has e^-0.2 of the mass
    loss, grad = calls(x, keep.int(), val, lse, temperature)
    near(loss, grad, exact(x, keep.int(), val, lse, temperature), vocab, temperature)


@pytest.mark.parametrize("rows,vocab", FORMS)
def test_unlisted_logits_of_the_types_lowest_value(rows, vocab):
    gen = torch.Generator("cuda").manual_seed(2)
    x = torch.full((rows, vocab), torch.finfo(torch.float32).min, device="cuda")
    x[:, :50] = torch.randn(rows, 50, device="cuda", generator=gen)
    idx = torch.arange(30, dtype=torch.int32, device="cuda").expand(rows, 30).contiguous()  # 20 of the others are unlisted too
    val = torch.randn(rows, 30, device="cuda", generator=gen)
    lse = torch.logsumexp(val.double(), dim=1).float() + 0.2
    for some in (x, torch.where(torch.arange(vocab, device="cuda") < 30, x, torch.finfo(torch.float32).min)):
        loss, grad = calls(some.contiguous(), idx, val, lse, 1.0)
        near(loss, grad, exact(some, idx, val, lse, 1.0), vocab)


def test_the_gradient_of_far_unlisted_logits_agrees_with_differences():
    """Central differences with step h: off by the third derivative (at most 1 for this loss) times h^2 / 6, and by the roundings of
    two losses of about 150, 2^-24 of each, and of the perturbed logits, 2^-24 of at most 256 (a slope of at most 1), over 2 h."""
    gen = torch.Generator("cuda").manual_seed(4)
    x = torch.randn(1, 40, device="cuda", generator=gen)
    x[:, 6:] -= 150.0
    idx = torch.arange(6, dtype=torch.int32, device="cuda")[None]
    val = torch.randn(1, 6, device="cuda", generator=gen)
    lse = torch.logsumexp(val.double(), dim=1).float() + 0.5
    h, n = 2.0 ** -4, 80
    eye = h * torch.eye(40, device="cuda")
    rows = torch.cat([x + eye, x - eye])
    loss = torch.empty(n, device="cuda")
    B.pvt_distill_loss(B.make_distill(rows, idx.expand(n, 6).contiguous(), val.expand(n, 6).contiguous(),
                                      teacher_lse=lse.expand(n).contiguous()), loss)
    slope = (loss[:40] - loss[40:]).double() / (2 * h)
    one, grad = torch.empty(1, device="cuda"), torch.empty(1, 40, device="cuda")
    B.pvt_distill_loss(B.make_distill(x, idx, val, teacher_lse=lse), one, grad=grad)
    noise = 2 * 256 * 2.0 ** -24 + 2 * 256 * 2.0 ** -24 + 4 * off(40)
    assert ((slope - grad[0].double()).abs() <= h * h / 6 + noise / (2 * h)).all()
    assert grad[0, 6:].sum().item() < -0.3  # the rest of the mass, 0.39, is asked for


def test_a_loss_near_nothing_with_the_remaining_mass():
    """A student that leaves almost nothing unlisted, as its teacher: the listed part of both sums is binary64, so the loss is off by
    the unlisted sum's own share of them."""
    vocab, k, rows = 3000, 4, 64
    gen = torch.Generator("cuda").manual_seed(6)
    teacher = torch.full((rows, vocab), -20.0, device="cuda")
    teacher[:, :k] = torch.randn(rows, k, device="cuda", generator=gen)
    student = teacher.clone()
    student[:, k:] += 0.3
    lse = torch.logsumexp(teacher.double(), dim=1).float()
    lse = torch.where(torch.arange(rows, device="cuda") % 2 == 0, lse, torch.nextafter(lse, torch.zeros_like(lse)))
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(rows, k).contiguous()
    val = teacher[:, :k].contiguous()
    want, _, q, _, unlisted = exact(student, idx, val, lse, 1.0)
    loss, _ = calls(student, idx, val, lse, 1.0)
    part = q[:, k:].sum(dim=1) + unlisted.sum(dim=1)
    assert ((loss.double() - want).abs() <= off(vocab) * part + 2.0 ** -24 * want.abs() + 1e-14).all()


def lse_noise(lse, p):
    """What may be left of 1 - sum p by the rounding of a binary32 teacher_lse and of its sum."""
    return p.sum(dim=1) * 2.0 ** -22 * (18 + lse.double().abs())


def list_alone(loss, grad, x, idx, val, lse, temperature):
    """Near the loss of the list alone.  With lse off by d every p is off by d of itself: the loss by d (1 + loss), the gradient by
    d (p + q)."""
    vocab = x.shape[1]
    want_loss, want_grad, q, p, _ = exact(x, idx, val, None, temperature)
    d = lse_noise(lse, p)
    e = off(vocab)
    assert torch.isfinite(loss).all()
    assert ((loss.double() - want_loss).abs() <= 2 * e + d * (1 + want_loss) + 2.0 ** -24 * want_loss.abs()).all()
    eps, tiny = torch.finfo(grad.dtype).eps / 2, torch.finfo(grad.dtype).tiny
    bound = (2 * e * q + 2.0 ** -23 * p + d[:, None] * (p + q)) / temperature + eps * want_grad.abs() + tiny * eps + 1e-37
    assert ((grad.double() - want_grad).abs() <= bound).all()


def teacher_lists(teacher, k, temperature):
    """A teacher's list, and its lse: as the list's call gives it, rounded from binary64, and its neighbours to both sides."""
    rows = teacher.shape[0]
    idx, val = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
    lse = torch.empty(rows, device="cuda")
    B.pvt_distill_top(teacher, idx, val, lse, temperature=temperature)
    t = torch.tensor(temperature).item()
    rounded = torch.logsumexp(teacher.double() / t, dim=1).float()
    up = torch.full_like(rounded, math.inf)
    return idx, val, [lse, rounded, torch.nextafter(rounded, up), torch.nextafter(rounded, -up)]


@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("shift", [0.0, -7.0, 300.0])
@pytest.mark.parametrize("rows,vocab", [(200, 40), (700, 130), (3, 1024)])
def test_a_list_of_the_whole_vocabulary_leaves_nothing(rows, vocab, shift, temperature):
    gen = torch.Generator("cuda").manual_seed(vocab)
    teacher = torch.randn(rows, vocab, device="cuda", generator=gen) * 2 + shift
    student = torch.randn(rows, vocab, device="cuda", generator=gen)
    idx, val, lses = teacher_lists(teacher, vocab, temperature)
    for lse in lses:
        loss, grad = calls(student, idx, val, lse, temperature)
        list_alone(loss, grad, student, idx, val, lse, temperature)
    far = lses[0] + 0.1  # whatever the lse says
    near(*calls(student, idx, val, far, temperature), exact(student, idx, val, far, temperature, rest=False), vocab, temperature)


MASKS = [-math.inf, -1e4, torch.finfo(torch.float32).min]


@pytest.mark.parametrize("student_mask", MASKS)
@pytest.mark.parametrize("teacher_mask", MASKS)
@pytest.mark.parametrize("k", [40, 64])
@pytest.mark.parametrize("rows,vocab,shift,temperature", [(200, 100, 0.0, 1.0), (700, 1000, 20.0, 0.7), (3, 66000, -7.0, 1.0)])
def test_a_mask_that_leaves_no_more_than_the_list(rows, vocab, shift, temperature, k, teacher_mask, student_mask):
    """40 entries are allowed, in teacher and student: the teacher's remaining mass is what rounding its lse leaves, and not asked of
    a student that has none."""
    gen = torch.Generator("cuda").manual_seed(vocab + k)
    allowed = torch.randperm(vocab, device="cuda", generator=gen)[:40]
    teacher = torch.full((rows, vocab), teacher_mask, device="cuda")
    teacher[:, allowed] = torch.randn(rows, 40, device="cuda", generator=gen) * 2 + shift
    student = torch.full((rows, vocab), student_mask, device="cuda")
    student[:, allowed] = torch.randn(rows, 40, device="cuda", generator=gen)
    idx, val, lses = teacher_lists(teacher, k, temperature)
    assert (idx[:, 40:] >= 0).all() == (k == 40 or teacher_mask > -math.inf)
    left = 0
    for lse in lses:
        loss, grad = calls(student, idx, val, lse, temperature)
        list_alone(loss, grad, student, idx[:, :40], val[:, :40], lse, temperature)
        p = torch.exp(val.double() / torch.tensor(temperature).item() - lse.double()[:, None])
        left += (p.sum(dim=1) < 1).sum().item()
    assert left > rows / 2  # (of 4 rows each: some of both kinds)


def test_a_rest_that_rounding_does_not_explain_is_asked_of_every_student():
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.full((5, 300), -math.inf, device="cuda")
    x[:, :20] = torch.randn(5, 20, device="cuda", generator=gen)
    idx = torch.arange(20, dtype=torch.int32, device="cuda").expand(5, 20).contiguous()
    val = torch.randn(5, 20, device="cuda", generator=gen)
    lse = torch.logsumexp(val.double(), dim=1).float() + 1e-3
    loss, grad = calls(x, idx, val, lse, 1.0)
    assert (loss == math.inf).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,vocab", FORMS)
def test_a_nan_that_is_listed_shows_in_the_whole_row(rows, vocab, tail):
    gen = torch.Generator("cuda").manual_seed(8)
    idx = torch.arange(40, dtype=torch.int32, device="cuda").expand(rows, 40).contiguous()
    val = torch.randn(rows, 40, device="cuda", generator=gen)
    lse = torch.logsumexp(val.double(), dim=1).float() + 0.1 if tail else None
    x = torch.randn(rows, vocab, device="cuda", generator=gen)
    x[0, 37] = math.nan
    for others in (x, torch.where(torch.arange(vocab, device="cuda") < 40, x, -math.inf)):
        loss, grad = calls(others.contiguous(), idx, val, lse, 1.0)
        assert torch.isnan(loss[0]) and torch.isnan(grad[0]).all()
        assert not torch.isnan(loss[1:]).any() and not torch.isnan(grad[1:]).any()
