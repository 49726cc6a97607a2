"""Sums of very many terms, and factors of zero."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


def policy(B, x, tokens, old, rf, adv, kl_coef, workers=1):
    shape = B.make_logits(workers, tokens.numel() // workers, x.shape[1], B.TYPE_F32)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    loss, kl, grad = torch.empty(workers, device="cuda"), torch.empty(workers, device="cuda"), torch.empty_like(x)
    B.dbw_policy_loss(shape, x, tokens, old, rf, adv, None, 0.2, 0.2, kl_coef, loss, work, kl_out=kl, dlogits=grad)
    return loss, kl, grad


def test_sums_of_very_many_rows(B):
    """Equal terms, whose roundings all have one sign."""
    rows = 1 << 20
    x, tokens, zero = torch.zeros(rows, 1, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
    adv = torch.full((rows,), -0.1, device="cuda")
    loss, _, _ = policy(B, x, tokens, zero, zero, adv, 0.0)
    assert abs(loss.item() / 0.1 - 1) < 4 * 2.0 ** -24
