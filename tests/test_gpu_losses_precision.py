"""How exact log-probabilities and preference margins are: errors of one sign would add up over a sequence.

With u = 2^-24, H = -sum p ln p <= ln V the entropy of a row, d = x - max x: a term's exponent is off by u |s d| (the rounding of d and that of the
product), 2^x by 2 u, and weighted with p that is u (H + 2) of ln Z; a sum of eight terms rounds three times, the lanes' sum once, the
logarithm once, and the result to 32 bits by u |log p|.  All of these go to the nearest value, so they have no common sign."""
import math

import numpy as np
import pytest
import torch

import loss_reference as ref

pytestmark = pytest.mark.gpu

U = ref.U
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


def logits_of(dtype, rows, vocab, seed):
    """A trained model's rows on the GPU: a broad floor of unlikely tokens, the given one often among the likely."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, vocab, device="cuda", generator=g) * 2
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    x[torch.arange(rows, device="cuda"), tokens] = torch.randn(rows, device="cuda", generator=g) * 4 + 8
    return x.to(dtype), tokens.int(), g


def exact_logp(x, tokens, scale):
    out = torch.empty(x.shape[0], dtype=torch.float64, device="cuda")
    for a in range(0, x.shape[0], 512):
        out[a:a + 512] = ref.token_logp(x[a:a + 512], tokens[a:a + 512], scale)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 0.8, 0.9, 1.25])
def test_log_probabilities_are_off_to_either_side(B, dtype, scale):
    rows, vocab = 8192, 20011
    x, tokens, _ = logits_of(dtype, rows, vocab, seed=int(100 * scale))
    shape = B.make_logits(1, rows, vocab, dtype, scale=scale)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    logp = torch.empty(rows, device="cuda")
    B.dbw_token_logp(shape, x, tokens, logp, work)
    want = exact_logp(x, tokens, scale)
    off = logp.double() - want
    assert (off.abs() <= U * (want.abs() + 2 * math.log(vocab) + 8)).all()
    # a log-probability of up to 16 is rounded by 2.8e-7 (root of the mean square), of a mean over 8192 by 3e-9
    assert abs(off.mean().item()) <= 2e-8, f"mean error {off.mean().item():.3g}"


# sequences of few and of many rows, whole or in slices, in pairs that the gradient's workgroups sum up by themselves
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,lengths,gradient", [(30011, [1000, 100], False), (70001, [600, 60], True), (9001, [40, 15, 12, 40], True), (300, [900, 20, 80, 700], True)])
def test_margins_of_ragged_sequences(B, dtype, vocab, lengths, gradient):
    rows, pairs, scale = sum(lengths), len(lengths) // 2, 0.9
    x, tokens, g = logits_of(dtype, rows, vocab, seed=vocab)
    want = exact_logp(x, tokens, scale)
    rf = (want + torch.randn(rows, device="cuda", generator=g) * 0.2).float()
    start = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device="cuda")
    shape = B.make_logits(1, rows, vocab, dtype, scale=scale)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    loss, margin, logp = torch.empty(1, device="cuda"), torch.empty(pairs, device="cuda"), torch.empty(rows, device="cuda")
    grad = torch.empty_like(x) if gradient else None
    B.dbw_preference_loss(shape, pairs, x, tokens, start, rf, None, 1.0, 0.0, loss, work, margin, logp_out=logp, dlogits=grad)
    assert ((logp.double() - want).abs() <= U * (want.abs() + 2 * math.log(vocab) + 8)).all()
    part = torch.split(want - rf.double(), lengths)
    for j in range(pairs):
        u = (part[2 * j].sum() - part[2 * j + 1].sum()).item()
        n = lengths[2 * j] + lengths[2 * j + 1]
        # a row's error before it is rounded to 32 bits is about u and has no common sign: six times the root of their number; of a
        # mean, 2e-9 a row (a tenth of what is allowed above)
        assert abs(margin[j].item() - u) <= 6 * math.sqrt(n) * U + 2e-9 * n + 2 * U * abs(u), f"pair {j}: {margin[j].item()} for {u}"
