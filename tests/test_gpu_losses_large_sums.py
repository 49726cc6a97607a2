"""The gradient from the log of a row's sum of exponentials, where that is a large number: rounded to 32 bits it has lost the logarithm of the sum."""
import math

import pytest
import torch

import loss_reference as ref
import test_gpu_losses as base

pytestmark = pytest.mark.gpu

U = ref.U
F32, BF16, F16 = base.F32, base.BF16, base.F16
B = base.B


def rows_of_all_sizes(I, dtype):
    """Logits of I's rows; rows from `bad` on have no distribution."""
    low = torch.finfo(dtype).min
    x = torch.randn(I.total, I.v, generator=I.g) * 2
    x[0] = low                                           # nothing but a mask of the type's lowest value
    x[1] = low
    x[1, I.v // 3:] = 1.0
    x[2] += 1024
    x[3] -= 300
    x[4] = torch.finfo(dtype).max / 4                    # equal, and large
    x[5] = x[5] * 30 - 20000
    x[6] = -math.inf
    x[6, [0, I.v - 1]] = torch.tensor([-5000.0, -5001.0])
    x[7] += 200                                          # its L is still taken as it is
    bad = 8
    x[8] = -math.inf
    x[9, I.v // 2] = math.inf
    x[10, I.v // 2] = math.nan
    return x.to(dtype), bad


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab,pad,shift", [(300, 1, 1), (3001, 0, 3), (20011, 5, 0), (100003, 0, 1)])
@pytest.mark.parametrize("scale", [1.0, 2.0])
def test_gradients_of_rows_with_large_sums(B, dtype, vocab, pad, shift, scale):
    I = base.Inputs(B, dtype, 1, 11, vocab, pad, shift, scale=scale)
    I.x, bad = rows_of_all_sizes(I, dtype)
    I.rows_of(I.flat).copy_(I.x)
    I.dev.copy_(I.flat)
    tokens = I.token_array()
    logp, lse, coef = torch.empty(11, device="cuda"), torch.empty(11, device="cuda"), torch.linspace(-1.5, 2, 11).cuda()
    B.dbw_token_logp(I.shape, I.logits(), tokens, logp, I.work, lse_out=lse)
    grad = I.gradient()
    B.dbw_token_logp_grad(I.shape, I.logits(), tokens, lse, coef, grad[I.shift:])
    got = I.rows_of(grad.cpu())
    for r in range(bad, 11):
        assert torch.isnan(got[r]).all(), f"row {r} has no distribution"
    z = ref.scaled(I.x[:bad], scale)
    lp = torch.log_softmax(z, 1)
    p = torch.exp(lp)
    y = torch.nn.functional.one_hot(I.tokens[:bad], vocab).double()
    c = coef.cpu().double()[:bad, None]
    want = torch.zeros(11, vocab, dtype=torch.float64)
    slack = torch.zeros_like(want)
    want[:bad] = scale * c * (y - p)
    # exponents of the terms that are not zero, the sum, and of an L up to 256 its rounding
    spread = torch.where(p > 0, (lp.amax(1, keepdim=True) - lp).clamp(max=110), 0.0)
    large = torch.logsumexp(z, 1).abs()
    rel = U * (4 * spread + 2 * math.log(vocab) + 40 + torch.where(large <= 256, 2 * large, 0.0)[:, None])
    slack[:bad] = scale * c.abs() * (p * rel + y * 4 * U)
    I.live[bad:] = False
    flat = grad.cpu()
    I.rows_of(flat)[bad:] = 0
    I.check_gradient(flat, want, slack)
    mine = I.dev.clone()                                 # in place
    B.dbw_token_logp_grad(I.shape, mine[I.shift:], tokens, lse, coef, mine[I.shift:])
    assert torch.equal(I.rows_of(mine)[:bad], I.rows_of(grad)[:bad])
