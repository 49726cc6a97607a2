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


@pytest.mark.parametrize("rows,vocab", [(4, 50), (100, 50), (4, 40001)])
def test_an_advantage_or_a_coefficient_of_zero_takes_its_term_out(B, rows, vocab):
    """However far a ratio or a reference's probability is beyond 32 bits."""
    x = torch.randn(rows, vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    logp = torch.log_softmax(x, 1)[:, 0]
    adv = torch.ones(rows, device="cuda")
    adv[0] = 0.0
    old = logp.clone()
    old[0] = -200.0                                      # a ratio of e^190
    loss, _, grad = policy(B, x, tokens, old, None, adv, 0.0)
    assert abs(loss.item() + (rows - 1) / rows) < 1e-5 and torch.isfinite(grad).all() and (grad[0] == 0).all()
    x[1, 0] = -150.0                                     # the reference finds the token likely, the model does not
    logp = torch.log_softmax(x.double(), 1)[:, 0].float()
    old, rf = logp.clone(), logp.clone()
    rf[1] = -1.0
    adv.fill_(1.0)
    loss, kl, grad = policy(B, x, tokens, old, rf, adv, 0.0)
    assert abs(loss.item() + 1) < 1e-4 and kl.item() == math.inf and torch.isfinite(grad).all()
    # a ratio that is no number stays one
    old[2] = math.nan
    adv[2] = 0.0
    loss, kl, grad = policy(B, x, tokens, old, rf, adv, 0.0)
    assert torch.isnan(loss).all() and torch.isnan(grad[2]).all() and torch.isfinite(grad[:2]).all()


def test_sums_of_very_many_rows(B):
    """Equal terms, whose roundings all have one sign."""
    rows = 1 << 20
    x, tokens, zero = torch.zeros(rows, 1, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
    adv = torch.full((rows,), -0.1, device="cuda")
    loss, _, _ = policy(B, x, tokens, zero, zero, adv, 0.0)
    assert abs(loss.item() / 0.1 - 1) < 4 * 2.0 ** -24
