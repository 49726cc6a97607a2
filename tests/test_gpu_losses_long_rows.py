"""Kernels that hold a row, on as many long rows as are not cut: workgroups of 512 threads, rows that are held in part, rows that go to the XCDs in an order of
their own; also in place, which gives the same bits."""
import pytest
import torch

import test_gpu_losses as base

pytestmark = pytest.mark.gpu

F32, BF16, F16 = base.F32, base.BF16, base.F16
B = base.B

# 24, 48, 64, 100 and 300 KB, one XCD's rows more than the others'
ROWS = [(F32, 3, 24, 6007), (BF16, 2, 36, 24007), (BF16, 3, 25, 32768), (F16, 1, 73, 50001), (F32, 2, 40, 25003), (BF16, 1, 75, 150001), (F32, 1, 66, 75001)]


@pytest.mark.parametrize("dtype,n,t,v", ROWS)
def test_policy(B, dtype, n, t, v):
    I = base.Inputs(B, dtype, n, t, v, pad=v % 2, shift=v % 5, left=3, scale=0.8)
    old, rf, adv = base.policy_inputs(I)
    grad = I.gradient()
    loss, kl, logp = base.run_policy(I, old, rf, adv, None, grad)
    base.check_policy(I, old, rf, adv, None, loss, kl, logp, grad)
    tokens, old, rf, adv, mine = I.token_array(), I.scattered(old), I.scattered(rf), I.scattered(adv), I.dev.clone()
    again = torch.empty_like(loss)
    B.dbw_policy_loss(I.shape, mine[I.shift:], tokens, old, rf, adv, None, 0.2, 0.28, 0.05, again, I.work, dlogits=mine[I.shift:])
    assert torch.equal(again, loss) and torch.equal(I.rows_of(mine), I.rows_of(grad))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,n,t,v", [(BF16, 2, 9, 32768), (F32, 1, 17, 17001), (F16, 1, 19, 150001)])
def test_distillation(B, dtype, n, t, v, tail):
    I = base.Inputs(B, dtype, n, t, v, pad=v % 2, shift=v % 5, scale=0.8, banned=7)
    index, value, lse = base.teacher_of(I, 100, tail)
    index = torch.where(index < v - 7, index, -1)
    index[:, 0] = torch.where((index >= 0).any(1), index[:, 0], I.tokens)
    if tail:
        lse = (torch.logsumexp(torch.where(index >= 0, base.ref.scaled(value, I.scale), -float("inf")), 1) + 0.2).float()
    grad, row_loss = I.gradient(), torch.full((I.total,), 7.0, device="cuda")
    loss = base.run_distill(I, index, value, lse, None, grad, row_loss)
    base.check_distill(I, index, value, lse, None, loss, row_loss, grad)
    mine = I.dev.clone()
    again = torch.empty_like(loss)
    B.dbw_distill_loss(I.shape, 100, mine[I.shift:], index.int().cuda(), value.cuda(), None, again, I.work,
                       teacher_lse=None if lse is None else lse.cuda(), dlogits=mine[I.shift:])
    assert torch.equal(again, loss) and torch.equal(I.rows_of(mine), I.rows_of(grad))
