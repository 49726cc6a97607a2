"""Preference losses of few rows in many pairs: on either side of where a gradient's workgroups sum the pairs up themselves."""
import pytest
import torch

import loss_reference as ref
import test_gpu_losses as base

pytestmark = pytest.mark.gpu

F32, BF16, F16 = base.F32, base.BF16, base.F16
B = base.B


@pytest.mark.parametrize("dtype,n,t,v,pairs", [(BF16, 1, 70, 500, 16), (F16, 1, 70, 500, 17), (F32, 32, 8, 300, 8), (F32, 33, 8, 300, 8), (BF16, 1, 1000, 260, 300)])
def test_many_pairs(B, dtype, n, t, v, pairs):
    I = base.Inputs(B, dtype, n, t, v, pad=1, left=1)
    rf = (ref.token_logp(I.x, I.tokens, I.scale) + torch.randn(I.total, generator=I.g)).float()
    start = base.cut(I.total, n, t, pairs, v)
    grad = I.gradient()
    loss, margin, logp = base.run_preference(I, start, rf, None, pairs, 0.3, 0.1, grad)
    base.check_preference(I, start, rf, None, pairs, 0.3, 0.1, loss, margin, logp, grad)
    again = base.run_preference(I, start, rf, None, pairs, 0.3, 0.1, None)
    for a, b in zip(again, (loss, margin, logp)):
        assert torch.equal(a, b)


def test_time_does_not_grow_with_the_number_of_pairs(B):
    I = base.Inputs(B, BF16, 1, 1000, 500)
    tokens, rf, grad = I.token_array(), torch.zeros(1000, device="cuda"), I.gradient()

    def best(pairs):
        start = torch.tensor(base.cut(1000, 1, 1000, pairs, 1), dtype=torch.int32, device="cuda")
        loss, margin, times = torch.empty(1, device="cuda"), torch.empty(pairs, device="cuda"), []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(20):
                B.dbw_preference_loss(I.shape, pairs, I.logits(), tokens, start, rf, None, 0.1, 0.0, loss, I.work, margin, dlogits=grad)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    assert best(500) < 4 * best(16)
