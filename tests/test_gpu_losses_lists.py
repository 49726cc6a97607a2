"""Distillation with long lists, also ones that repeat a column: what is reported and which entry counts."""
import pytest
import torch

import test_gpu_losses as base

pytestmark = pytest.mark.gpu

F32, BF16, F16 = base.F32, base.BF16, base.F16
B = base.B


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,n,t,v,k", [(BF16, 1, 70, 1000, 700), (F16, 1, 3, 1001, 1000), (F32, 2, 3, 500, 400), (BF16, 1, 80, 600, 200), (F32, 1, 2, 9001, 1024),
                                           (BF16, 1, 70, 690, 334), (F32, 1, 3, 400, 337)])      # 64 KB of lists a workgroup
def test_long_lists(B, dtype, n, t, v, k, tail):
    I = base.Inputs(B, dtype, n, t, v, pad=1, scale=0.8)
    index, value, lse = base.teacher_of(I, k, tail)
    grad, row_loss = I.gradient(), torch.full((I.total,), 7.0, device="cuda")
    loss = base.run_distill(I, index, value, lse, None, grad, row_loss)
    base.check_distill(I, index, value, lse, None, loss, row_loss, grad)
    assert I.status.item() == B.OK


@pytest.mark.parametrize("dtype,t,v,k", [(F32, 6, 300, 64), (BF16, 80, 300, 64), (BF16, 3, 1000, 700), (F32, 70, 2000, 500), (F16, 3, 33001, 1024),
                                         (BF16, 3, 70001, 1000)])
def test_lists_that_are_filled_up_with_a_repeated_column(B, dtype, t, v, k):
    """The first entry of a column counts, wherever the others stand."""
    I = base.Inputs(B, dtype, 1, t, v)
    index, value, _ = base.teacher_of(I, k, False, short=False)
    filled, taken = index.clone(), index.clone()
    for r in range(t):
        if r % 3 == 0:                                   # a short list, filled up with its first entry, or with its last
            filled[r, 5:], taken[r, 5:] = index[r, 0], -1
        elif r % 3 == 1:
            filled[r, 40:], taken[r, 40:] = index[r, 39], -1
        else:                                            # every column twice, the second time in another order
            half = k // 2
            filled[r, half:2 * half], taken[r, half:2 * half] = index[r, :half].flip(0), -1
    grad, row_loss = I.gradient(), torch.full((t,), 7.0, device="cuda")
    loss = base.run_distill(I, filled, value, None, None, grad, row_loss)
    assert I.status.item() == B.ERR_INVALID
    base.check_distill(I, taken, value, None, None, loss, row_loss, grad)


def test_a_repeated_column_does_not_hold_up_the_call(B):
    """As many comparisons as pairs of entries at most, shared by a row's threads: a few times the time of a list of distinct columns, not a thousand."""
    I = base.Inputs(B, F16, 1, 512, 8200)
    index, value, _ = base.teacher_of(I, 1024, False, short=False)
    filled = index.clone()
    filled[:, 512:] = index[:, :512].flip(1)
    value, loss, grad = value.cuda(), torch.empty(1, device="cuda"), I.gradient()

    def best(list_):
        list_, times = list_.int().cuda(), []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            B.dbw_distill_loss(I.shape, 1024, I.logits(), list_, value, None, loss, I.work, dlogits=grad)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    assert best(filled) < 30 * best(index)
