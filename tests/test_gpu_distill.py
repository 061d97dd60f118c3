"""A teacher's top logits and the loss against them, against float64."""
import math

import pytest
import torch

import student_reference as ref
from paper_2405_14852_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def top(logits, k, temperature=1.0):
    rows = logits.shape[0]
    idx = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    val, lse = torch.full((rows, k), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    B.pvt_distill_top(logits, idx, val, lse, temperature=temperature)
    return idx, val, lse


def check_top(logits, k, temperature=1.0):
    idx, val, lse = top(logits, k, temperature)
    want_idx, want_val, want_lse = ref.top(logits, k, temperature)
    assert torch.equal(idx.long(), want_idx)
    assert torch.equal(torch.isnan(val), torch.isnan(want_val))
    assert (torch.isnan(val) | (val.double() == want_val)).all()
    fine = torch.isfinite(want_lse)
    assert torch.equal(torch.isnan(lse), torch.isnan(want_lse))
    assert torch.equal(lse[~fine & ~torch.isnan(lse)].double(), want_lse[~fine & ~torch.isnan(want_lse)])
    # exponents are off by at most 2^-23 of themselves (two roundings) and terms by 2^-22 of ex2: relative to a term y <= 1 that
    # is |log y| y 2^-23 < 2^-24, so the sum of n terms, added in chains of at most n / 512 + 16 + 8 roundings, is off by
    # less than (n / 512 + 40) 2^-24 + n 2^-24 / sum of it; a bound on its logarithm, and two roundings of the result
    n = logits.shape[1]
    err = (lse.double() - want_lse).abs()[fine]
    z = torch.exp(want_lse - logits.double().amax(dim=1) / temperature)[fine]
    bound = 2.0 ** -23 * (n / 512 + 60) + 2.0 ** -23 * want_lse[fine].abs() + 2.0 ** -22 * (torch.log(z.clamp(min=1)) + 4)
    assert (err <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 7, 7), (2, 500, 62), (5, 1000, 1), (300, 1001, 64), (2, 5000, 1024),
                                          (1, 32000, 64), (4, 50001, 300), (3, 131071, 257), (1, 262144, 1000), (700, 4099, 100)])
def test_top_logits(rows, vocab, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(vocab + k)
    logits = (2.5 * torch.randn(rows, vocab, device="cuda", generator=gen)).to(dtype)
    check_top(logits, k)
    check_top(logits, k, 2.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 2), (7, 9)])
def test_top_logits_of_rows_of_any_alignment(offset, pad, dtype):
    wide = torch.randn(9, offset + 3001 + pad, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
    wide[:, :offset] = 1e4
    wide[:, offset + 3001:] = 1e4
    check_top(wide[:, offset:offset + 3001], 50)


@pytest.mark.parametrize("rows,vocab", [(2, 3000), (1, 70000), (400, 5000)])
def test_ties_go_to_the_lowest_index(rows, vocab):
    same = torch.zeros(rows, vocab, device="cuda")
    check_top(same, 100)
    few = torch.randint(0, 3, (rows, vocab), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).float()
    check_top(few, 513)
    few[:, vocab // 2] = -0.0
    few[few == 0] = -0.0
    few[:, vocab // 3] = 0.0
    check_top(-few, 700)
    close = 20.0 + torch.rand(rows, vocab, device="cuda", generator=torch.Generator("cuda").manual_seed(2)) * 1e-3
    check_top(close, 300)


@pytest.mark.parametrize("vocab", [2000, 90000])
def test_masked_and_special_logits(vocab):
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(10, vocab, device="cuda", generator=gen)
    x[0, 37:] = -math.inf          # fewer than k are left
    x[1, :] = -math.inf            # none
    x[2, 100:] = torch.finfo(torch.float32).min
    x[3, 5] = math.inf
    x[3, 900] = math.inf
    x[4, 7] = math.nan
    x[5, 7] = math.nan
    x[5, 1000] = math.inf
    x[5, 1500] = math.nan
    x[6, :] = torch.finfo(torch.float32).min
    x[7, ::2] = -math.inf
    x[8, :] = -math.inf
    x[8, vocab - 1] = -3.0
    x[9, :] = -1e4
    x[9, 0] = 1e4
    check_top(x, 64)


def problem(rows, vocab, k, dtype, seed, pad=0, near=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    teacher = 2.5 * torch.randn(rows, vocab, device="cuda", generator=gen)
    wide = torch.full((rows, vocab + pad), 1e4, device="cuda").to(dtype)
    student = wide[:, :vocab]
    student.copy_(0.9 * teacher + near * torch.randn(rows, vocab, device="cuda", generator=gen))
    val, idx = torch.topk(teacher, k, dim=1)
    return student, idx.int(), val.contiguous(), teacher


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k,temperature,pad", [(1, 2, 1, 1.0, 0), (3, 33, 5, 1.0, 0), (5, 1000, 64, 2.0, 3),
                                                          (2, 5003, 1024, 0.7, 0), (400, 777, 20, 1.0, 7), (2, 40000, 200, 1.0, 8),
                                                          (1, 131071, 300, 3.0, 1)])
def test_loss_and_gradient(rows, vocab, k, temperature, pad, dtype, tail):
    x, idx, val, teacher = problem(rows, vocab, k, dtype, vocab + rows, pad)
    lse = torch.logsumexp(teacher.double() / temperature, dim=1).float() if tail else None
    gen = torch.Generator(device="cuda").manual_seed(8)
    weight = torch.rand(rows, device="cuda", generator=gen)
    if rows > 2:
        weight[1] = 0.0
    up = torch.rand(rows, device="cuda", generator=gen) + 0.5
    want_loss, want_grad = ref.distill(x, idx, val, lse, weight, up, temperature)
    want_loss, want_grad = want_loss.cuda(), want_grad.cuda()
    d = B.make_distill(x, idx, val, teacher_lse=lse, weight=weight, temperature=temperature)
    loss, stats = torch.full((rows,), math.nan, device="cuda"), torch.full((rows, 8), math.nan, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    grad = torch.full((rows, vocab), math.nan, dtype=dtype, device="cuda")
    B.pvt_distill_loss(d, loss, upstream=up, grad=grad, status=status)
    # a probability is off by at most e of itself, e = 2^-23 (n / 1024 + 40): 2^-22 of ex2, |log y| 2^-23 of the exponent
    # (|log y| y sums to less than 20 of the sum here) and n / 512 + 24 roundings of sums; its logarithm by e.  The loss is a mean
    # of logarithms under weights that add up to 1, the gradient a difference of two probabilities or shares.
    e = 2.0 ** -23 * (vocab / 1024 + 40)
    assert ((loss.double() - want_loss).abs() <= weight.double() * (2 * e + 2.0 ** -24 * want_loss.abs() / weight.clamp(min=1e-9))).all()
    q = torch.softmax(x.double() / temperature, dim=1)
    factor = (weight * up).double()[:, None] / temperature
    p = torch.zeros_like(q)
    norm = torch.logsumexp(val.double() / temperature, dim=1) if lse is None else lse.double()
    p.scatter_(1, idx.long(), torch.exp(val.double() / temperature - norm[:, None]))
    share = q.scatter(1, idx.long(), 0.0)
    share = share / share.sum(dim=1, keepdim=True).clamp(min=1e-300) * (1 - p.sum(dim=1, keepdim=True)).clamp(min=0) if tail else 0 * share
    eps = torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 2.0 ** -24
    # (below the smallest normal number of the type a rounding is half of the smallest number)
    bound = factor * (2 * e * (q + share) + 2.0 ** -23 * p) + eps * want_grad.abs() + torch.finfo(dtype).tiny * eps + 1e-38
    assert ((grad.double() - want_grad).abs() <= bound).all()

    # the same in two calls, in place, in another type
    B.pvt_distill_loss(d, loss, stats=stats, status=status)
    again = torch.full((rows, vocab), math.nan, dtype=dtype, device="cuda")
    B.pvt_distill_grad(d, stats, again, upstream=up, status=status)
    assert torch.equal(again, grad)
    f32 = torch.full((rows, vocab + 1), 3.0, device="cuda")
    B.pvt_distill_grad(d, stats, f32[:, 1:], upstream=up, status=status)
    assert torch.equal(f32[:, 1:].to(dtype), grad) and (f32[:, 0] == 3).all()
    both = loss.clone()
    keep = x.clone()
    B.pvt_distill_grad(d, stats, x, upstream=up, status=status)
    assert torch.equal(x, grad)
    x.copy_(keep)
    B.pvt_distill_loss(d, loss, upstream=up, grad=x, stats=stats, status=status)
    assert torch.equal(x, grad) and torch.equal(loss, both)
    if pad:
        wide = x._base if x._base is not None else x
        assert (wide[:, vocab:].float() == torch.tensor(1e4).to(dtype).float()).all()
    assert status.item() == 0


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_agrees_with_differences_of_the_loss(tail):
    """Central differences with step h: off by the third derivative (at most 1 for this loss) times h^2 / 6, and by the loss's
    own error, 2 * 2^-23 * 40, over 2 h."""
    x, idx, val, teacher = problem(1, 40, 6, torch.float32, 5)
    lse = torch.logsumexp(teacher.double(), dim=1).float() if tail else None
    h = 2.0 ** -5
    rows = torch.cat([x + h * torch.eye(40, device="cuda"), x - h * torch.eye(40, device="cuda")])
    n = rows.shape[0]
    d = B.make_distill(rows, idx.expand(n, 6).contiguous(), val.expand(n, 6).contiguous(),
                       teacher_lse=None if lse is None else lse.expand(n).contiguous())
    loss = torch.empty(n, device="cuda")
    B.pvt_distill_loss(d, loss)
    slope = (loss[:40] - loss[40:]).double() / (2 * h)
    grad, one = torch.empty(1, 40, device="cuda"), torch.empty(1, device="cuda")
    B.pvt_distill_loss(B.make_distill(x, idx, val, teacher_lse=lse), one, grad=grad)
    # (perturbed inputs are rounded too: 2^-24 of at most 16, times a slope of at most 1)
    assert ((slope - grad[0].double()).abs() <= h * h / 6 + (4 * 2.0 ** -23 * 40 + 2.0 ** -20) / (2 * h)).all()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("vocab", [600, 66000])
def test_rows_without_effect_and_masked_logits(vocab, tail):
    k, rows = 8, 9
    x, idx, val, teacher = problem(rows, vocab, k, torch.float32, 6)
    lse = torch.logsumexp(teacher.double(), dim=1).float() if tail else None
    weight = torch.ones(rows, device="cuda")
    idx[0] = -1                                   # nothing is listed
    idx[1, 3:] = -1                               # a shorter list
    val[2] = -math.inf                            # nothing above -infinity is listed
    val[3, 4:] = -math.inf
    x[4] = -math.inf                              # the student's mask leaves nothing
    weight[5] = 0.0
    x[5] = math.nan
    x[6] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, -math.inf, x[6])
    x[6].scatter_(0, idx[6].long(), 0.5)
    x[7].scatter_(0, idx[7, :1].long(), torch.full((1,), -math.inf, device="cuda"))  # an infinite loss, a gradient that is not
    x[8] = torch.finfo(torch.float32).min         # a mask of the type's lowest value: a uniform student
    want_loss, want_grad = ref.distill(x, idx, val, lse, weight)
    d = B.make_distill(x, idx, val, teacher_lse=lse, weight=weight)
    loss, grad = torch.empty(rows, device="cuda"), torch.empty(rows, vocab, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pvt_distill_loss(d, loss, grad=grad, status=status)
    e = 2.0 ** -23 * (vocab / 1024 + 40)
    assert (loss[[0, 2, 4, 5]] == 0).all() and (grad[[0, 2, 4, 5]] == 0).all()
    assert loss[7].item() == math.inf and torch.isfinite(grad[7]).all()
    some = [1, 3, 6, 8]
    assert ((loss[some].cpu().double() - want_loss[some]).abs() <= 2 * e + 2.0 ** -24 * want_loss[some].abs()).all()
    assert ((grad.cpu().double() - want_grad).abs() <= 4 * e).all()
    assert status.item() == 0


def test_bad_and_repeated_entries_are_left_out_and_reported():
    vocab, k = 1000, 600
    x, idx, val, _ = problem(4, vocab, k, torch.float32, 7)
    idx[1, 0] = vocab
    idx[1, 5] = 2 ** 31 - 1
    idx[2, 7] = idx[2, 3]
    idx[2, 500] = idx[2, 3]
    idx[2, 599] = idx[2, 0]
    idx[3, 9] = -5
    want_loss, want_grad = ref.distill(x, idx, val)
    for rows, flag in (([0, 3], 0), ([1], B.PVT_DEV_BAD_INDEX), ([2], B.PVT_DEV_BAD_INDEX)):
        n = len(rows)
        d = B.make_distill(x[rows], idx[rows].contiguous(), val[rows].contiguous())
        loss, grad, stats = torch.empty(n, device="cuda"), torch.empty(n, vocab, device="cuda"), torch.empty(n, 8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.pvt_distill_loss(d, loss, grad=grad, stats=stats, status=status)
        assert status.item() == flag
        assert ((loss.cpu().double() - want_loss[rows]).abs() <= 1e-5).all()  # 2^-23 * 41 * 2 of a mean of logarithms
        assert ((grad.cpu().double() - want_grad[rows]).abs() <= 1e-5).all()
        again = torch.empty(n, vocab, device="cuda")
        B.pvt_distill_grad(d, stats, again)
        assert torch.equal(again, grad)


def test_nan_and_infinite_student_logits_show():
    x, idx, val, _ = problem(3, 500, 5, torch.float32, 9)
    x[0, 400] = math.nan
    x[1, 400] = math.inf
    d = B.make_distill(x, idx, val)
    loss, grad = torch.empty(3, device="cuda"), torch.empty(3, 500, device="cuda")
    B.pvt_distill_loss(d, loss, grad=grad)
    assert torch.isnan(loss[0]) and torch.isnan(grad[0]).all()
    assert not torch.isfinite(loss[1])
    assert torch.isfinite(loss[2]) and torch.isfinite(grad[2]).all()


def test_a_student_near_its_teacher_keeps_the_rest_s_gradient():
    """Listed probabilities that leave 1e-6 of the mass: differences of sums would lose the rest."""
    vocab, k = 3000, 4
    teacher = torch.full((1, vocab), -20.0, device="cuda")
    teacher[0, :k] = torch.tensor([1.0, 0.5, 0.0, -0.5])
    student = teacher.clone()
    student[0, k:] += 0.3
    lse = torch.logsumexp(teacher.double(), dim=1).float()
    idx, val = torch.arange(k, dtype=torch.int32, device="cuda")[None], teacher[:, :k].contiguous()
    _, want = ref.distill(student, idx, val, lse)
    d = B.make_distill(student, idx, val, teacher_lse=lse)
    loss, grad = torch.empty(1, device="cuda"), torch.empty(1, vocab, device="cuda")
    B.pvt_distill_loss(d, loss, grad=grad)
    want = want.cuda()[0, k:]
    # the teacher's rest hangs on the rounding of its lse, which the formula shares: only the kernel's own errors count
    assert ((grad[0, k:].double() - want).abs() <= 2.0 ** -23 * 64 * want.abs() + 1e-16).all()


def test_captured_steps_share_nothing():
    x, idx, val, _ = problem(6, 9000, 32, torch.bfloat16, 10)
    keep = x.clone()
    d = B.make_distill(x, idx, val)
    loss, grad = torch.zeros(6, device="cuda"), torch.zeros(6, 9000, dtype=torch.bfloat16, device="cuda")
    loss2, grad2 = torch.zeros_like(loss), torch.zeros_like(grad)
    B.pvt_distill_loss(d, loss, grad=grad)
    want = loss.clone(), grad.clone()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g, (l, gr) in zip(graphs, ((loss, grad), (loss2, grad2))):
        with torch.cuda.graph(g):
            B.pvt_distill_loss(d, l, grad=gr)
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, st in zip(graphs, side):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(grad, want[1]) and torch.equal(loss2, want[0]) and torch.equal(grad2, want[1])
    x.copy_(keep + 1)
    graphs[0].replay()
    torch.cuda.synchronize()
    # (a shift of all logits: rounding of bfloat16 aside nothing changes)
    assert ((loss - want[0]).abs() <= 0.1).all()


def test_rows_further_apart_than_32_bits_count():
    rows, vocab, k, apart = 3, 5000, 30, 2 ** 31 + 8
    x = torch.empty(2 * apart + 8192, dtype=torch.bfloat16, device="cuda").as_strided((rows, vocab), (apart, 1))
    x.copy_(torch.randn(rows, vocab, device="cuda", generator=torch.Generator("cuda").manual_seed(3)))
    near = x.clone(memory_format=torch.contiguous_format).contiguous()
    outs = []
    for logits in (x, near):
        idx, val, lse = (torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda"),
                         torch.empty(rows, device="cuda"))
        B.pvt_distill_top(logits, idx, val, lse=lse)
        d = B.make_distill(logits, idx, val * 0.5, teacher_lse=lse)
        loss = torch.empty(rows, device="cuda")
        B.pvt_distill_loss(d, loss, grad=logits)
        outs.append((idx, val, lse, loss, logits))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k", [(700, 500, 20), (700, 1042, 33), (650, 2051, 128), (600, 3001, 200), (1200, 7, 5)])
def test_many_short_rows(rows, vocab, k, dtype):
    """Blocks of few threads, each with a row."""
    x, idx, val, teacher = problem(rows, vocab, k, dtype, vocab, 1)
    special = x.clone()
    special[3] = 1.5
    special[5, : vocab // 2] = -math.inf
    special[6] = -math.inf
    check_top(special, k, 1.3)
    check_top(x, k, 1.3)
    n, temperature = 12, 1.3
    for lse in (None, torch.logsumexp(teacher.double() / temperature, dim=1).float()):
        d = B.make_distill(x, idx, val, teacher_lse=lse, temperature=temperature)
        loss, grad = torch.empty(rows, device="cuda"), torch.empty(rows, vocab, dtype=dtype, device="cuda")
        B.pvt_distill_loss(d, loss, grad=grad)
        assert torch.isfinite(loss).all() and torch.isfinite(grad).all()
        want_loss, want_grad = ref.distill(x[:n], idx[:n], val[:n], None if lse is None else lse[:n], None, None, temperature)
        want_loss, want_grad = want_loss.cuda(), want_grad.cuda()
        # as above: a probability is off by e of itself, the rest of the student's mass carries the rest of the teacher's
        e = 2.0 ** -23 * (vocab / 1024 + 40)
        assert ((loss[:n].double() - want_loss).abs() <= 2 * e + 2.0 ** -24 * want_loss.abs()).all()
        eps = torch.finfo(dtype).eps / 2
        bound = 2 * e * 2 / temperature + eps * want_grad.abs() + torch.finfo(dtype).tiny * eps
        assert ((grad[:n].double() - want_grad).abs() <= bound).all()
        stats, again = torch.empty(rows, 8, device="cuda"), torch.empty_like(grad)
        B.pvt_distill_loss(d, loss, stats=stats)
        B.pvt_distill_grad(d, stats, again)
        assert torch.equal(again, grad)
