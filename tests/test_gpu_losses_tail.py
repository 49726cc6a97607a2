"""Distillation with the teacher's whole mass given: the class of everything outside its list, where that is far less likely than the list, where the teacher's
rest is small, and where nothing lies outside."""
import math

import pytest
import torch

import loss_reference as ref
import test_gpu_losses as base

pytestmark = pytest.mark.gpu

U = ref.U
F32, BF16, F16 = base.F32, base.BF16, base.F16
B = base.B


def expected(I, index, value, lse):
    """Row losses, gradients over w, and bounds on the error of either, from 64 bits.  The class outside is taken by itself: S as a difference of logarithms,
    its gradient (S - R) times the distribution within the class."""
    z = ref.scaled(I.x, I.scale)
    t = ref.scaled(value, I.scale)
    inside = torch.zeros(I.x.shape, dtype=torch.bool).scatter_(1, index, True)
    lp = torch.log_softmax(z, 1)
    out = z.masked_fill(inside, -math.inf)
    log_s = torch.logsumexp(out, 1) - torch.logsumexp(z, 1)
    some = torch.isfinite(log_s)
    within = torch.where(some[:, None], torch.softmax(torch.where(some[:, None], out, 0.0), 1), 0.0)
    log_q = t - lse.double()[:, None]
    q = torch.exp(log_q)
    rest = (1 - q.sum(1)).clamp(min=0)
    at = lp.gather(1, index)
    # log q is rounded once and raised with two roundings more; the sums are wider
    rel_q = U * (log_q.abs() + 4)
    d_rest = (q * rel_q).sum(1) + U * rest
    use = some & (rest > 0)
    over = torch.where(use, torch.log(torch.where(use, rest, 1.0)) - torch.where(use, log_s, 0.0), 0.0)
    loss = (q * (log_q - at)).sum(1) + rest * over
    rel_p = U * (at.abs() * 2 + 2 * math.log(I.v) + 16)
    d_loss = (q * (rel_q * ((log_q - at).abs() + 1) + rel_p)).sum(1) + torch.where(use, d_rest * (over.abs() + 1), 0.0) + 8 * U * loss.abs() + 16 * U * (rest * over).abs()
    s = float(torch.tensor(I.scale).float())
    grad = s * torch.where(some, torch.exp(log_s) - rest, 0.0)[:, None] * within
    # within the class: exponents of up to max |s d| over it
    spread = torch.where(within > 0, (out.amax(1, keepdim=True) - out).clamp(max=200), 0.0)
    d_grad = s * within * ((torch.exp(log_s) + rest)[:, None] * U * (2 * spread + 2 * math.log(I.v) + 40) + d_rest[:, None])
    grad.scatter_(1, index, s * (torch.exp(at) - q))
    d_grad.scatter_(1, index, s * (torch.exp(at) * rel_p + q * rel_q))
    return loss, d_loss, grad, d_grad


def check(I, index, value, lse, what=""):
    row_loss, grad = torch.full((I.total,), 7.0, device="cuda"), I.gradient()
    loss = base.run_distill(I, index, value, lse, None, grad, row_loss)
    want, d_want, g, d_g = expected(I, index, value, lse)
    base.close(row_loss, want, d_want, f"{what}: row losses")
    base.close(loss, want.reshape(I.n, I.t).mean(1), d_want.reshape(I.n, I.t).mean(1) + 16 * U * want.abs().reshape(I.n, I.t).mean(1), f"{what}: loss")
    I.check_gradient(grad, g / I.t, d_g / I.t, what)
    assert I.status.item() == I.B.OK
    return loss


def prepared(B, dtype, rows, vocab, k, scale, seed):
    I = base.Inputs(B, dtype, 1, rows, vocab, scale=scale, seed=seed, peak=0.0)
    index = torch.stack([torch.randperm(vocab, generator=I.g)[:k] for _ in range(rows)])
    return I, index


def student(I, x):
    I.x = x.to(I.dtype)
    I.rows_of(I.flat).copy_(I.x)
    I.dev.copy_(I.flat)


# a worker's rows in one workgroup, rows of 16 and of 64 threads, of a workgroup, of a workgroup that holds part of them
SIZES = [(6, 300, 5), (70, 300, 5), (5, 1900, 20), (70, 1900, 20), (3, 10007, 64), (2, 70001, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,k", SIZES)
@pytest.mark.parametrize("offset", [0.0, 30.0, -300.0])
def test_a_small_rest_of_a_teacher_whose_logits_are_far_from_zero(B, dtype, rows, vocab, k, offset):
    I, index = prepared(B, dtype, rows, vocab, k, 0.9, seed=5)
    student(I, torch.randn(rows, vocab, generator=I.g))
    value = torch.randn(rows, k, generator=I.g) + offset
    lse = (torch.logsumexp(ref.scaled(value, 0.9), 1) - math.log(0.99)).float()
    check(I, index, value, lse, f"offset {offset}")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,vocab,k", SIZES)
def test_everything_outside_the_list_far_below_it(B, dtype, rows, vocab, k):
    for scale, gap in ((0.5, 85.0), (1.0, 90.0), (1.0, 120.0), (10.0, 95.0), (0.7, None)):
        I, index = prepared(B, dtype, rows, vocab, k, scale, seed=int(gap or 1))
        x = torch.randn(rows, vocab, generator=I.g)
        if gap is None:
            outside = torch.ones(rows, vocab, dtype=torch.bool).scatter_(1, index, False)
            x = x.masked_fill(outside, torch.finfo(dtype).min)
        else:
            x = x / scale
            x.scatter_add_(1, index, torch.full(index.shape, gap / scale))
        student(I, x)
        value = torch.randn(rows, k, generator=I.g)
        lse = (torch.logsumexp(ref.scaled(value, scale), 1) - math.log(0.9)).float()
        check(I, index, value, lse, f"scale {scale}, gap {gap}")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,vocab,k", [(40, 40, 40), (70, 300, 300), (40, 1000, 1000), (60, 1900, 20), (40, 10007, 64), (8, 70001, 128)])
@pytest.mark.parametrize("offset", [0.0, 200.0])
def test_nothing_outside_the_list(B, dtype, rows, vocab, k, offset):
    """The list is the whole vocabulary, or no other token can occur; the teacher's L is that of its list, rounded: no row or its gradient is infinite."""
    I, index = prepared(B, dtype, rows, vocab, k, 0.9, seed=6)
    x = torch.randn(rows, vocab, generator=I.g)
    outside = torch.ones(rows, vocab, dtype=torch.bool).scatter_(1, index, False)
    student(I, x.masked_fill(outside, -math.inf))
    value = torch.randn(rows, k, generator=I.g) + offset
    lse = torch.logsumexp(ref.scaled(value, 0.9), 1).float()
    loss = check(I, index, value, lse)
    assert torch.isfinite(loss).all()
    # a rest that is no rounding: infinitely dear, and a token that cannot occur has no gradient
    row_loss, grad = torch.empty(rows, device="cuda"), I.gradient()
    base.run_distill(I, index, value, lse + 0.01, None, grad, row_loss)
    assert (row_loss == math.inf).all()
    got = I.rows_of(grad).cpu()
    assert torch.isfinite(got).all() and (got[outside] == 0).all()
