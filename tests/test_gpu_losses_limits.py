"""The losses on logits at the limits of their header: the most workers, pairs and rows."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
MOST = 1 << 22                                           # workers, and pairs of all workers


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


def test_the_most_pairs(B):
    rows, vocab = 1025, 5
    x = torch.randn(rows, vocab, device="cuda")
    tokens = torch.randint(0, vocab, (rows,), device="cuda").int()
    start = torch.zeros(2 * MOST + 1, dtype=torch.int32, device="cuda")
    start[-2], start[-1] = 1000, rows                    # the last pair has all rows
    shape = B.make_logits(1, rows, vocab, B.TYPE_F32)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    loss, margin, grad = torch.empty(1, device="cuda"), torch.full((MOST,), 7.0, device="cuda"), torch.empty_like(x)
    B.dbw_preference_loss(shape, MOST, x, tokens, start, torch.zeros(rows, device="cuda"), None, 0.01, 0.0, loss, work, margin, dlogits=grad)
    lp = torch.log_softmax(x.double(), 1)
    logp = lp.gather(1, tokens.long()[:, None])[:, 0]
    u = 0.01 * float(logp[:1000].sum() - logp[1000:].sum())
    assert not margin[:-1].any() and abs(margin[-1].item() - u) < 1e-5 * abs(u)
    want = ((MOST - 1) * math.log(2) + math.log1p(math.exp(-u))) / MOST
    assert abs(loss.item() - want) < 2.0 ** -23
    slope = -0.01 / MOST / (1 + math.exp(u))
    want = -torch.exp(lp)
    want[torch.arange(rows), tokens.long()] += 1
    want *= slope
    want[1000:] *= -1
    assert ((grad.double() - want).abs() <= 2e-5 * want.abs() + 1e-6 * abs(slope)).all()


def test_the_most_workers_in_one_workgroup_each(B):
    rows, vocab, total = 64, 2, MOST * 64                # 1024 threads each
    x = torch.zeros(total, vocab, dtype=BF16, device="cuda")
    tokens = torch.zeros(total, dtype=torch.int32, device="cuda")
    shape = B.make_logits(MOST, rows, vocab, BF16)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    loss, grad = torch.full((MOST,), 7.0, device="cuda"), torch.full_like(x, 7.0)
    old, adv = torch.full((total,), -math.log(2), device="cuda"), torch.ones(total, device="cuda")
    adv[-rows:] = 2.0
    B.dbw_policy_loss(shape, x, tokens, old, None, adv, None, 0.2, 0.2, 0.0, loss, work, dlogits=grad)
    assert ((loss[:-1] + 1).abs() < 1e-6).all() and abs(loss[-1].item() + 2) < 1e-6
    want = torch.tensor([-0.5, 0.5], device="cuda") / rows
    assert torch.equal(grad[:-rows], want.to(BF16).expand(total - rows, 2)) and torch.equal(grad[-rows:], (2 * want).to(BF16).expand(rows, 2))
    del old, adv
    grad.fill_(7.0)
    loss.fill_(7.0)
    B.dbw_distill_loss(shape, 1, x, tokens, torch.zeros(total, device="cuda"), None, loss, work, dlogits=grad)
    assert ((loss - math.log(2)).abs() < 1e-6).all()
    assert torch.equal(grad, want.to(BF16).expand(total, 2))


def test_the_most_rows(B):
    """Row numbers up to 2^31 - 2, in steps of a workgroup's threads."""
    rows, vocab, pairs, last = (1 << 31) - 1, 2, 2048, 1500
    x = torch.zeros(rows * vocab, dtype=BF16, device="cuda")
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    shape = B.make_logits(1, rows, vocab, BF16)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    rf = torch.full((rows,), -math.log(2), device="cuda")
    rf[-last:] = -1.0
    start = torch.linspace(0, rows - last, 2 * pairs, dtype=torch.float64).long()
    start = torch.cat([start, torch.tensor([rows])]).int().cuda()           # the last sequence: the last rows
    loss, margin = torch.full((1,), 7.0, device="cuda"), torch.full((pairs,), 7.0, device="cuda")
    grad = torch.full_like(x, 7.0)
    B.dbw_preference_loss(shape, pairs, x, tokens, start, rf, None, 0.01, 0.0, loss, work, margin, dlogits=grad)
    u = -0.01 * last * (1 - math.log(2))
    assert (margin[:-1].abs() < 1e-3).all() and abs(margin[-1].item() - u) < 1e-3
    slope = lambda u: -0.01 / pairs / (1 + math.exp(u))
    tail = grad[-2 * last:].view(last, 2).double().cpu()
    want = torch.tensor([-0.5, 0.5], dtype=torch.float64) * slope(u)
    assert ((tail - want).abs() <= 2.0 ** -7 * want.abs()).all()
    head = grad[:2000].view(1000, 2).double().cpu()
    want = torch.tensor([0.5, -0.5], dtype=torch.float64) * slope(0.0)
    assert ((head - want).abs() <= 2.0 ** -7 * want.abs()).all()
    del grad, start
    B.dbw_policy_loss(shape, x, tokens, rf, None, torch.ones(rows, device="cuda"), None, 0.2, 10.0, 0.0, loss, work)
    want = -((rows - last) + last * math.e / 2) / rows
    assert abs(loss.item() - want) < 1e-6
