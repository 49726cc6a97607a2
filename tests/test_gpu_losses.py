"""The losses on logits against the same in 64 bits (loss_reference.py): types, odd sizes, strides and starts, rows that take no part
whatever they hold, empty lists and sequences, tokens that cannot occur, in place, other streams, captured calls."""
import math

import numpy as np
import pytest
import torch

import loss_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


class Inputs:
    """Logits of `workers` times `rows` rows in a larger array: `pad` elements between rows, `shift` before the first.  Every element that
    is not a live row's is NaN; `left` rows of each worker take no part, `banned` columns of the others cannot occur."""

    def __init__(self, B, dtype, workers, rows, vocab, pad=0, shift=0, scale=1.0, left=0, banned=0, seed=0, peak=6.0):
        g = torch.Generator().manual_seed(seed * 1000003 + vocab)
        self.B, self.dtype, self.n, self.t, self.v = B, dtype, workers, rows, vocab
        self.scale, self.ld, self.shift = scale, vocab + pad, shift
        total = self.total = workers * rows
        x = torch.randn(total, vocab, generator=g) * 2
        self.tokens = torch.randint(0, max(1, vocab - banned), (total,), generator=g)
        x[torch.arange(total), self.tokens] += peak * torch.rand(total, generator=g)
        if banned:
            x[:, vocab - banned:] = -math.inf
        self.x = x.to(dtype)
        self.live = torch.ones(total, dtype=torch.bool)
        for i in range(workers):
            self.live[i * rows + torch.randperm(rows, generator=g)[:left]] = False
        self.g = g
        flat = torch.full((shift + total * self.ld + 8,), math.nan, dtype=dtype)
        view = self.rows_of(flat)
        view[self.live] = self.x[self.live]
        self.flat = flat
        self.shape = B.make_logits(workers, rows, vocab, dtype, ld=self.ld, scale=scale)
        self.dev = flat.cuda()
        self.tol = torch.where(self.live, ref.tol(self.x, scale), 0.0)
        self.work = torch.empty(B.dbw_loss_work_bytes(self.shape), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def rows_of(self, flat):
        return flat[self.shift:self.shift + self.total * self.ld].view(self.total, self.ld)[:, :self.v]

    def logits(self):
        return self.dev[self.shift:]

    def gradient(self):
        """An array for the gradient, all of it a mark that no gradient has."""
        return torch.full_like(self.dev, 77.0)

    def token_array(self):
        return torch.where(self.live, self.tokens, -1 - torch.arange(self.total) % 3).int().cuda()

    def scattered(self, v, fill=math.nan):
        return torch.where(self.live, v.double(), fill).float().cuda()

    def check_gradient(self, dev, want, slack, what=""):
        """want [total, V] in 64 bits, slack [total, V]: bound on the error before the one rounding to the type."""
        got = dev.cpu()
        outside = torch.ones_like(got, dtype=torch.bool)
        self.rows_of(outside)[:] = False
        assert (got[outside].float() == 77.0).all(), f"{what}: written beyond the rows"
        got = self.rows_of(got).double()
        assert (got[~self.live] == 0).all(), f"{what}: rows that take no part"
        bound = slack * 1.001 + ref.HALF_ULP[self.dtype] * (want.abs() + slack) + ref.SUBNORMAL[self.dtype]
        bad = ~((got - want).abs() <= bound)
        assert not bad[self.live].any(), (f"{what}: {int(bad[self.live].sum())} of {bad[self.live].numel()} elements, worst "
                                          f"{((got - want).abs() / bound)[self.live].max():.3g} of the bound")


def close(got, want, bound, what=""):
    got, want = got.detach().cpu().double(), want.double()
    bound = bound + ref.U * 4 * want.abs() + 1e-37
    assert ((got - want).abs() <= bound).all(), f"{what}: {((got - want).abs() / bound).max():.3g} of the bound"


# sizes around what a lane, a wave and a workgroup hold at once, one column, and rows of many workgroups' worth
VOCABS = [1, 2, 7, 64, 65, 259, 1000, 4099, 8192, 33001]
SHAPES = [(F32, 3, 5, 257, 0, 0), (BF16, 2, 7, 1000, 0, 0), (F16, 1, 3, 4097, 3, 1), (F32, 2, 2, 33001, 1, 3), (BF16, 1, 4, 50000, 8, 0),
          (BF16, 3, 3, 20011, 5, 7), (F16, 2, 2, 65536, 0, 0), (BF16, 1, 2, 131072, 0, 0), (F32, 1, 2, 131073, 2, 1),
          (BF16, 1, 2, 300001, 0, 3), (BF16, 2, 64, 512, 0, 0), (F32, 1, 65, 129, 1, 0), (BF16, 1, 17, 4097, 0, 1), (F32, 3, 31, 2049, 0, 0),
          (F16, 1, 256, 8200, 1, 0), (BF16, 257, 1, 8200, 0, 1), (F32, 5, 51, 4100, 0, 2), (BF16, 1, 1, 131072, 0, 0), (F16, 40, 9, 130, 2, 1), (BF16, 1, 1, 9, 0, 0), (F32, 1, 1, 1, 4, 1), (F32, 2, 300, 33, 0, 0)]


# --------------------------------------------------------------------------- log-probabilities

def run_logp(I):
    logp, lse = torch.full((I.total,), 7.0, device="cuda"), torch.full((I.total,), 7.0, device="cuda")
    I.B.dbw_token_logp(I.shape, I.logits(), I.token_array(), logp, I.work, lse_out=lse, status_out=I.status)
    return logp, lse


def want_logp(I):
    want, lse = torch.zeros(I.total, dtype=torch.float64), torch.zeros(I.total, dtype=torch.float64)
    want[I.live] = ref.token_logp(I.x, I.tokens, I.scale)[I.live]
    lse[I.live] = torch.logsumexp(ref.scaled(I.x, I.scale), 1)[I.live]
    return want, lse


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_log_probabilities_and_their_gradient(B, dtype, vocab):
    I = Inputs(B, dtype, 2, 5, vocab, pad=vocab % 3, shift=vocab % 2, scale=0.7, left=1, banned=vocab // 9)
    logp, lse = run_logp(I)
    want, want_lse = want_logp(I)
    close(logp, want, I.tol, "logp")
    close(lse, want_lse, I.tol + 2 * ref.U * want_lse.abs(), "lse")
    coef = torch.randn(I.total, generator=I.g)
    grad = I.gradient()
    coef_dev = I.scattered(coef)                        # NaN where the token is negative
    B.dbw_token_logp_grad(I.shape, I.logits(), I.token_array(), lse, coef_dev, grad[I.shift:], status_out=I.status)
    check_logp_gradient(I, grad, coef.double(), torch.zeros(I.total), extra=4 * ref.U * (want_lse.abs() + 1))
    assert I.status.item() == B.OK


def check_logp_gradient(I, grad, coef, coef_slack, extra=0.0, what="gradient"):
    p = torch.exp(ref.log_softmax(I.x, I.scale))
    d = -p
    d[torch.arange(I.total), I.tokens] += 1
    s = float(np.float32(I.scale))
    want = torch.where(I.live[:, None], s * coef[:, None] * d, 0.0)
    rel = (I.tol + extra + 8 * ref.U)[:, None]
    hot = p.clone()
    hot[torch.arange(I.total), I.tokens] += 1           # the two terms at the token cancel: roundings of either
    slack = s * (coef.abs()[:, None] * hot * rel + coef_slack[:, None].double() * (d.abs() + hot * rel))
    I.check_gradient(grad, want, slack, what)


@pytest.mark.parametrize("dtype,n,t,v,pad,shift", SHAPES)
def test_log_probabilities_over_shapes(B, dtype, n, t, v, pad, shift):
    I = Inputs(B, dtype, n, t, v, pad, shift, left=min(1, t - 1))
    logp, lse = run_logp(I)
    want, want_lse = want_logp(I)
    close(logp, want, I.tol, "logp")
    close(lse, want_lse, I.tol + 2 * ref.U * want_lse.abs(), "lse")
    only = torch.full((I.total,), 7.0, device="cuda")
    B.dbw_token_logp(I.shape, I.logits(), I.token_array(), only, I.work)
    assert torch.equal(only, logp)


def test_logits_of_all_sizes_and_impossible_tokens(B):
    """Logits far from zero, of the type's lowest and largest values, -inf in most places; rows of nothing but -inf, with +inf or NaN."""
    for dtype in TYPES:
        low, high = torch.finfo(dtype).min, min(torch.finfo(dtype).max, 1e30)
        I = Inputs(B, dtype, 1, 9, 3001, seed=1)
        x = I.rows_of(I.flat)
        x[0] = -math.inf
        x[0, I.tokens[0]] = 2.5                          # certain
        x[1] = low                                       # a mask of the type's lowest value: uniform where nothing else is
        x[2] = low
        x[2, I.tokens[2]] = 1.0
        x[3] += 2.0 ** 10
        x[4] = -math.inf
        x[5, 17] = math.inf
        x[6, 2900] = math.nan
        x[7, :] = high
        x[8] = -math.inf
        x[8, [5, 2000, int(I.tokens[8])]] = torch.tensor([1.0, 2.0, 3.0], dtype=dtype)
        I.dev.copy_(I.flat)
        tokens = I.token_array()
        logp, lse = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
        B.dbw_token_logp(I.shape, I.logits(), tokens, logp, I.work, lse_out=lse)
        want = ref.token_logp(x, I.tokens, 1.0)
        assert torch.isnan(logp[[4, 5, 6]]).all() and torch.isnan(want[[4, 5, 6]]).all()
        rest = [0, 1, 2, 3, 7, 8]
        bound = ref.tol(torch.where(torch.tensor([[0], [1], [1], [0], [1], [0]], dtype=torch.bool), torch.tensor(0.0), x[rest].float()), 1.0)
        close(logp[rest], want[rest], bound + 2 * ref.U * want[rest].abs(), str(dtype))
        coef = torch.ones(9, device="cuda")
        grad = I.gradient()
        I.live[[4, 5, 6]] = False
        B.dbw_token_logp_grad(I.shape, I.logits(), tokens, torch.where(I.live.cuda(), lse, 0.0), torch.where(I.live.cuda(), coef, 0.0), grad)
        got = I.rows_of(grad.cpu()).double()
        p = torch.exp(ref.log_softmax(x, 1.0))
        assert (got[[0, 2]].abs() <= 8 * ref.U * 2.5).all()  # certain tokens: L, its base and the exponential are each rounded
        for r in (8,):
            want = -p[r]
            want[I.tokens[r]] += 1
            assert ((got[r] - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all()
            assert (got[r][p[r] == 0] == 0).all()


def test_a_token_beyond_the_vocabulary_is_reported(B):
    I = Inputs(B, F32, 1, 4, 50)
    tokens = torch.tensor([3, 50, 7, 1 << 30], dtype=torch.int32, device="cuda")
    logp = torch.empty(4, device="cuda")
    B.dbw_token_logp(I.shape, I.logits(), tokens, logp, I.work, status_out=I.status)
    assert I.status.item() == B.ERR_INVALID
    close(logp, ref.token_logp(I.x, tokens.cpu().clamp(max=49), 1.0), I.tol)
    I.status.zero_()
    tokens.fill_(-5)
    B.dbw_token_logp(I.shape, I.logits(), tokens, logp, I.work, status_out=I.status)
    assert I.status.item() == B.OK and (logp == 0).all()


# --------------------------------------------------------------------------- distillation

def teacher_of(I, k, tail, seed=0, value_type=F32, short=True):
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(I.v, generator=g)[:k] for _ in range(I.total)])
    index[::2, 0] = torch.where((index[::2] == I.tokens[::2, None]).any(1), index[::2, 0], I.tokens[::2])
    if short and k > 1:
        index[1::3, k // 2:] = -1 - (torch.arange(k - k // 2) % 2)
    value = (torch.randn(I.total, k, generator=g) * 2).to(value_type)
    there = index >= 0
    lse = None
    if tail:
        t = torch.where(there, ref.scaled(value, I.scale), -math.inf)
        lse = (torch.logsumexp(t, 1) - torch.log(1 - (0.01 + 0.4 * torch.rand(I.total, generator=g).double()))).float()
    return index, value, lse


def run_distill(I, index, value, lse, weights, dlogits, row_loss=None):
    loss = torch.full((I.n,), 7.0, device="cuda")
    I.B.dbw_distill_loss(I.shape, index.shape[1], I.logits(), index.int().cuda(), value.cuda(), None if weights is None else weights.cuda(),
                         loss, I.work, teacher_lse=None if lse is None else lse.cuda(), row_loss_out=row_loss,
                         dlogits=None if dlogits is None else dlogits[I.shift:], status_out=I.status)
    return loss


def check_distill(I, index, value, lse, weights, loss, row_loss, grad):
    live = I.live
    w = (torch.full((I.total,), 1.0 / I.t) if weights is None else weights).double()
    x = I.x[live].double().requires_grad_()
    rows = ref.distill_rows(x, index[live], value[live], I.scale, None if lse is None else lse[live])
    (g,) = torch.autograd.grad((w[live] * rows).sum(), x)
    s = float(np.float32(I.scale))
    # errors: log p by tol, q by that of the teacher's figures; a loss has sum q (|log q| + |log p|) of them.  The rest's mass
    # 1 - sum q is off by 2 (k + |t|) u at most, and enters times the log of its ratio, and over the student's
    lp = ref.log_softmax(I.x[live], I.scale)
    p = torch.exp(lp)
    there = index[live] >= 0
    at = torch.where(there, index[live], 0)
    t = torch.where(there, ref.scaled(value[live], I.scale), -math.inf)
    norm = torch.logsumexp(t, 1) if lse is None else lse[live].double()
    log_q = t - norm[:, None]
    q = torch.exp(log_q)
    zt = torch.where(there, t.abs(), 0.0)
    zt = torch.where(torch.isinf(zt), 0.0, zt).amax(1) + norm.abs()
    rel_q = ref.U * (8 * zt + index.shape[1] / 64 + 32)
    tol = I.tol[live]
    mag = torch.where(q > 0, q * ((log_q - lp.gather(1, at)).abs() + 1), 0.0).sum(1)
    row_bound = mag * (rel_q + tol) + 2 * tol + 2 * rel_q
    slack_p, slack_q = (tol + rel_q + 8 * ref.U)[:, None] * p, torch.zeros_like(p)
    if lse is not None:
        inside = torch.zeros(p.shape[0], I.v + 1, dtype=torch.bool)
        inside.scatter_(1, torch.where(there, at, I.v), True)
        inside = inside[:, :-1]
        mass = torch.where(inside, 0.0, p).sum(1)
        rest = (1 - q.sum(1)).clamp(min=0)
        d_rest = 2 * rel_q + 2 * ref.U * index.shape[1]
        ratio = torch.where(rest > 0, rest / mass, 0.0)
        row_bound = row_bound + d_rest * (torch.where(rest > 0, torch.log(ratio.clamp(min=1e-300)).abs(), 0.0) + 2) + rest * 4 * tol
        d_ratio = d_rest / mass.clamp(min=1e-300) + ratio * 4 * tol
        slack_p = slack_p * (1 + ratio)[:, None] + torch.where(inside, 0.0, p * d_ratio[:, None])
    slack_q.scatter_add_(1, at, torch.where(there, q * (rel_q + 8 * ref.U)[:, None], 0.0))
    bound = torch.zeros(I.total, dtype=torch.float64)
    want_rows = torch.zeros(I.total, dtype=torch.float64)
    bound[live], want_rows[live] = row_bound, rows.detach()
    if row_loss is not None:
        close(row_loss, want_rows, bound, "row losses")
    sums = lambda a: a.reshape(I.n, I.t).sum(1)
    wl = torch.where(live, w, 0.0)
    close(loss, sums(wl * want_rows), sums(wl.abs() * bound) + 16 * ref.U * sums((wl * want_rows).abs()), "loss")
    if grad is not None:
        want, slack = torch.zeros(I.total, I.v, dtype=torch.float64), torch.zeros(I.total, I.v, dtype=torch.float64)
        want[live] = g
        slack[live] = s * w[live].abs()[:, None] * (slack_p + slack_q)
        I.check_gradient(grad, want, slack, "gradient")


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,k", [(1, 1), (2, 1), (7, 7), (64, 3), (259, 64), (1000, 65), (4099, 1), (8192, 1000), (33001, 128)])
def test_distillation(B, dtype, tail, vocab, k):
    if tail and k == vocab:
        tail = False                                     # nothing lies outside: its own test
    I = Inputs(B, dtype, 2, 4, vocab, pad=vocab % 4, shift=vocab % 3, scale=0.5, left=1, banned=vocab // 20 if k < vocab // 2 else 0)
    index, value, lse = teacher_of(I, k, tail, value_type=dtype)
    index = torch.where(index < vocab - (vocab // 20 if k < vocab // 2 else 0), index, -1)     # no teacher wants what cannot occur
    index[:, 0] = torch.where((index >= 0).any(1), index[:, 0], I.tokens)
    if tail:
        t = torch.where(index >= 0, ref.scaled(value, I.scale), -math.inf)
        lse = (torch.logsumexp(t, 1) + 0.3).float()
    weights = torch.where(I.live, 0.25 + torch.rand(I.total, generator=I.g), 0.0)
    row_loss, grad = torch.full((I.total,), 7.0, device="cuda"), I.gradient()
    loss = run_distill(I, index, value, lse, weights, grad, row_loss)
    check_distill(I, index, value, lse, weights, loss, row_loss, grad)
    assert I.status.item() == B.OK
    again = run_distill(I, index, value, lse, weights, None)
    assert torch.equal(again, loss)                      # the loss alone


@pytest.mark.parametrize("dtype,n,t,v,pad,shift", SHAPES)
def test_distillation_over_shapes(B, dtype, n, t, v, pad, shift):
    I = Inputs(B, dtype, n, t, v, pad, shift)
    k = min(33, (v + 1) // 2)
    index, value, lse = teacher_of(I, k, v > 2)
    grad = I.gradient()
    loss = run_distill(I, index, value, lse, None, grad)
    check_distill(I, index, value, lse, None, loss, None, grad)


def test_distillation_lists_that_leave_nothing_and_lists_of_everything(B):
    I = Inputs(B, F32, 1, 6, 40, seed=4)
    index = torch.arange(40).repeat(6, 1)
    value = torch.randn(6, 40, generator=I.g)
    index[1] = -1                                        # no list
    value[2] = -math.inf                                 # a list of impossible tokens
    value[3, 1:] = -math.inf                             # certain of one token
    index[4, 1:] = -1                                    # one entry
    I.live[1] = False
    I.live[2] = False
    row_loss, grad = torch.full((6,), 7.0, device="cuda"), I.gradient()
    loss = run_distill(I, index, value, None, None, grad, row_loss)
    check_distill(I, index, value, None, None, loss, row_loss, grad)
    # with the teacher's whole mass given, -inf entries leave the rest, which is everything outside: all of it for row 2's
    # list of the first 20 tokens; nothing lies outside row 0's
    I.live[2] = True
    I.dev.copy_(I.flat)
    I.rows_of(I.dev)[2] = I.x[2].cuda()
    index[2, 20:] = -1
    lse = torch.logsumexp(torch.where(index >= 0, value, -math.inf).double(), 1).float()
    lse[[1, 2]] = 0.0
    lse[0] -= 0.0
    value[0] -= 1e-3                                     # a little mass outside everything: infinitely dear
    loss = run_distill(I, index, value, lse, None, grad, row_loss)
    assert row_loss[0].item() == math.inf and loss.item() == math.inf
    assert row_loss[1].item() == 0 and (I.rows_of(grad)[1] == 0).all()
    p = torch.softmax(I.x[2].double(), 0)
    assert abs(row_loss[2].item() + math.log(p[20:].sum())) < 1e-5
    want = p.clone()
    want[20:] = p[20:] - p[20:] / p[20:].sum()
    assert (I.rows_of(grad)[2].cpu().double() - want / 6).abs().max() < 1e-6     # a weight of 1 / T


def test_distillation_a_student_almost_certain_of_the_teachers_tokens(B):
    """The student's mass outside the teacher's list far below fp32's resolution of one."""
    for dtype in TYPES:
        I = Inputs(B, dtype, 1, 3, 2000, seed=9)
        x = I.rows_of(I.flat)
        index = torch.stack([torch.randperm(2000, generator=I.g)[:8] for _ in range(3)])
        x[torch.arange(3)[:, None], index] += 40
        I.x = x.clone()
        I.dev.copy_(I.flat)
        I.tol = ref.tol(I.x, 1.0)
        value = torch.randn(3, 8, generator=I.g)
        lse = torch.logsumexp(value.double(), 1).float() + 0.1
        row_loss, grad = torch.empty(3, device="cuda"), I.gradient()
        loss = run_distill(I, index, value, lse, None, grad, row_loss)
        check_distill(I, index, value, lse, None, loss, row_loss, grad)


def test_distillation_reports_indices_that_do_not_belong(B):
    I = Inputs(B, F32, 1, 3, 100)
    index = torch.tensor([[4, 9, 4, 9], [100, 3, 1 << 30, 6], [8, 7, 6, 5]])
    value = torch.randn(3, 4, generator=I.g)
    grad, row_loss = I.gradient(), torch.empty(3, device="cuda")
    loss = run_distill(I, index, value, None, None, grad, row_loss)
    assert I.status.item() == B.ERR_INVALID
    taken = torch.tensor([[4, 9, -1, -1], [-1, 3, -1, 6], [8, 7, 6, 5]])        # the first of a column; none beyond the vocabulary
    check_distill(I, taken, value, None, None, loss, row_loss, grad)


# --------------------------------------------------------------------------- policy

def policy_inputs(I, with_ref=True):
    base = ref.token_logp(I.x, I.tokens, I.scale)
    step = torch.randn(I.total, generator=I.g).double() * 0.3
    for bound in (math.log(0.8), math.log(1.28)):        # the derivative jumps there
        step = torch.where((step - bound).abs() < 0.01, bound + 0.02, step)
    old = (base - step).float()
    rf = (base + torch.randn(I.total, generator=I.g) * 0.3).float() if with_ref else None
    return old, rf, torch.randn(I.total, generator=I.g)


def run_policy(I, old, rf, adv, weights, dlogits, tokens=None):
    loss, kl, logp = (torch.full((m,), 7.0, device="cuda") for m in (I.n, I.n, I.total))
    I.B.dbw_policy_loss(I.shape, I.logits(), I.token_array() if tokens is None else tokens, I.scattered(old),
                        None if rf is None else I.scattered(rf), I.scattered(adv), None if weights is None else weights.cuda(), 0.2, 0.28,
                        0.05, loss, I.work, kl_out=kl, logp_out=logp, dlogits=None if dlogits is None else dlogits[I.shift:],
                        status_out=I.status)
    return loss, kl, logp


def check_policy(I, old, rf, adv, weights, loss, kl, logp, grad):
    w = torch.where(I.live, (torch.full((I.total,), 1.0 / I.t) if weights is None else weights).double(), 0.0)
    base = torch.where(I.live, ref.token_logp(I.x, I.tokens, I.scale), 0.0)
    at = base.clone().requires_grad_()
    rows, kls = ref.policy_rows(at, torch.where(I.live, old, 0.0), None if rf is None else torch.where(I.live, rf, 0.0), adv, 0.2, 0.28, 0.05)
    (slope,) = torch.autograd.grad((w * rows).sum(), at)
    close(logp, base, I.tol, "logp")
    # rho and exp(d) are off by the log-probability's error, the difference's (2 u each of the terms) and the exponential's
    e = I.tol + 4 * ref.U * (base.abs() + old.abs() + (0 if rf is None else rf.abs()) + 2)
    rho = torch.exp(base - old.double())
    gone = torch.exp(rf.double() - base) if rf is not None else torch.zeros_like(base)
    d_kl = (gone + 1) * e
    d_row = rho * adv.abs() * e * 1.3 + 0.05 * d_kl + 4 * ref.U * rows.detach().abs()
    d_slope = w.abs() * (rho * adv.abs() * e + 0.05 * gone * e) * 1.01 + 4 * ref.U * slope.abs()
    sums = lambda a: a.reshape(I.n, I.t).sum(1)
    rows = rows.detach()
    close(loss, sums(w * rows), sums(w.abs() * d_row) + 16 * ref.U * sums((w * rows).abs()), "loss")
    close(kl, sums(w * kls.detach()), sums(w.abs() * d_kl) + 16 * ref.U * sums((w * kls.detach()).abs()), "kl")
    if grad is not None:
        check_logp_gradient(I, grad, slope, d_slope)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_policy(B, dtype, vocab):
    I = Inputs(B, dtype, 3, 4, vocab, pad=vocab % 2, shift=vocab % 3, scale=1.25, left=1, banned=vocab // 7)
    old, rf, adv = policy_inputs(I, with_ref=vocab != 64)
    weights = torch.where(I.live, torch.randn(I.total, generator=I.g), 0.0) if vocab % 2 else None
    grad = I.gradient()
    loss, kl, logp = run_policy(I, old, rf, adv, weights, grad)
    check_policy(I, old, rf, adv, weights, loss, kl, logp, grad)
    assert I.status.item() == B.OK
    again = run_policy(I, old, rf, adv, weights, None)
    for a, b in zip(again, (loss, kl, logp)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,n,t,v,pad,shift", SHAPES)
def test_policy_over_shapes(B, dtype, n, t, v, pad, shift):
    I = Inputs(B, dtype, n, t, v, pad, shift, left=min(1, t - 1))
    old, rf, adv = policy_inputs(I)
    grad = I.gradient()
    loss, kl, logp = run_policy(I, old, rf, adv, None, grad)
    check_policy(I, old, rf, adv, None, loss, kl, logp, grad)


def test_policy_rows_of_weight_zero_take_no_part(B):
    I = Inputs(B, BF16, 2, 6, 777, left=3)
    old, rf, adv = policy_inputs(I)
    weights = torch.where(I.live, 0.5, 0.0)
    grad = I.gradient()
    tokens = I.tokens.int().cuda()                       # every token is there; the weight alone leaves the row out
    loss, kl, logp = run_policy(I, old, rf, adv, weights, grad, tokens=tokens)
    check_policy(I, old, rf, adv, weights, loss, kl, logp, grad)


# --------------------------------------------------------------------------- preference

def run_preference(I, start, rf, weights, pairs, beta, smoothing, dlogits):
    loss, margin, logp = (torch.full((m,), 7.0, device="cuda") for m in (I.n, max(1, I.n * pairs), I.total))
    I.B.dbw_preference_loss(I.shape, pairs, I.logits(), I.token_array(), torch.tensor(start, dtype=torch.int32, device="cuda"),
                            I.scattered(rf), None if weights is None else weights.cuda(), beta, smoothing, loss, I.work, margin,
                            logp_out=logp, dlogits=None if dlogits is None else dlogits[I.shift:], status_out=I.status)
    return loss, margin[:I.n * pairs], logp


def check_preference(I, start, rf, weights, pairs, beta, smoothing, loss, margin, logp, grad):
    w = torch.where(I.live, (torch.ones(I.total) if weights is None else weights).double(), 0.0)
    base = torch.where(I.live, ref.token_logp(I.x, I.tokens, I.scale), 0.0)
    at = base.clone().requires_grad_()
    rf0 = torch.where(I.live, rf, 0.0)
    want, u = ref.preference(at, rf0, w, start, beta, smoothing, I.n, pairs)
    (slope,) = torch.autograd.grad(want.sum(), at)
    close(logp, base, I.tol, "logp")
    # a pair's sum adds a thread's rows / 64 + 10 terms, each off by the log-probability's error and a rounding of either term
    term = w.abs() * (I.tol + 2 * ref.U * (base.abs() + rf0.abs()))
    size = (w * (base - rf0.double())).abs()
    du = []
    for j in range(I.n * pairs):
        a, b = start[2 * j], start[2 * j + 2]
        du.append(abs(beta) * (term[a:b].sum() + ref.U * ((b - a) / 64 + 12) * size[a:b].sum()))
    du = torch.stack(du) + 2 * ref.U * u.detach().abs()
    close(margin, u.detach(), du, "margins")
    close(loss, want.detach(), (du + 8 * ref.U * (u.detach().abs() + 1)).reshape(I.n, pairs).sum(1) / pairs, "loss")
    if grad is not None:
        d_slope = torch.zeros(I.total, dtype=torch.float64)
        for j in range(I.n * pairs):
            a, b = start[2 * j], start[2 * j + 2]
            d_slope[a:b] = w[a:b].abs() * abs(beta) / pairs * (0.25 * du[j] + 8 * ref.U)
        check_logp_gradient(I, grad, slope, d_slope)


def cut(total, n, t, pairs, seed):
    g = np.random.default_rng(seed)
    start = []
    for i in range(n):
        start += [i * t] + sorted(int(c) for c in g.integers(0, t + 1, 2 * pairs - 1) + i * t)
    return start + [total]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,t,pairs,smoothing", [(1, 4, 1, 0.0), (7, 9, 2, 0.1), (259, 40, 3, 0.0), (1000, 12, 8, 0.5), (4099, 7, 1, 0.1),
                                                      (33001, 3, 1, 0.0)])
def test_preference(B, dtype, vocab, t, pairs, smoothing):
    I = Inputs(B, dtype, 2, t, vocab, pad=vocab % 2, shift=vocab % 3, scale=0.9, left=1)
    rf = (ref.token_logp(I.x, I.tokens, I.scale) + torch.randn(I.total, generator=I.g)).float()
    weights = torch.where(I.live, 0.1 + torch.rand(I.total, generator=I.g), 0.0) if vocab % 2 else None
    start = cut(I.total, 2, t, pairs, vocab)
    grad = I.gradient()
    loss, margin, logp = run_preference(I, start, rf, weights, pairs, 0.3, smoothing, grad)
    check_preference(I, start, rf, weights, pairs, 0.3, smoothing, loss, margin, logp, grad)
    assert I.status.item() == B.OK
    again = run_preference(I, start, rf, weights, pairs, 0.3, smoothing, None)
    for a, b in zip(again, (loss, margin, logp)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,n,t,v,pad,shift", SHAPES)
def test_preference_over_shapes(B, dtype, n, t, v, pad, shift):
    I = Inputs(B, dtype, n, t, v, pad, shift)
    rf = (ref.token_logp(I.x, I.tokens, I.scale) + torch.randn(I.total, generator=I.g)).float()
    start = cut(I.total, n, t, 1, v)
    grad = I.gradient()
    loss, margin, logp = run_preference(I, start, rf, None, 1, 0.5, 0.0, grad)
    check_preference(I, start, rf, None, 1, 0.5, 0.0, loss, margin, logp, grad)


@pytest.mark.parametrize("dtype,n,t,v,pairs", [(BF16, 3, 70, 500, 1), (BF16, 2, 65, 24000, 1), (F32, 2, 64, 12289, 1), (BF16, 2, 129, 300, 1), (F16, 1, 1030, 120, 20),
                                               (F32, 7, 9, 2100, 9)])
def test_preference_pairs_of_many_and_of_few_rows(B, dtype, n, t, v, pairs):
    """Either side of where a gradient's workgroups sum the pairs up themselves."""
    I = Inputs(B, dtype, n, t, v, pad=3, left=2)
    rf = (ref.token_logp(I.x, I.tokens, I.scale) + torch.randn(I.total, generator=I.g)).float()
    start = cut(I.total, n, t, pairs, v)
    start[0] += 1                                        # the first row in no sequence
    start = [max(s, 1) for s in start]
    grad = I.gradient()
    loss, margin, logp = run_preference(I, start, rf, None, pairs, 0.2, 0.05, grad)
    check_preference(I, start, rf, None, pairs, 0.2, 0.05, loss, margin, logp, grad)
    again = run_preference(I, start, rf, None, pairs, 0.2, 0.05, None)
    for a, b in zip(again, (loss, margin, logp)):
        assert torch.equal(a, b)


def test_preference_empty_sequences_gaps_and_large_margins(B):
    I = Inputs(B, F32, 1, 10, 60)
    rf = torch.zeros(10)
    base = ref.token_logp(I.x, I.tokens, 1.0)
    # rows 0, 1 and 9 in no sequence; an empty pair; a pair of one sequence; a margin that leaves no slope in fp32
    start = [2, 2, 2, 5, 5, 8, 9]
    grad = I.gradient()
    loss, margin, logp = run_preference(I, start, rf, None, 3, 200.0, 0.0, grad)
    check_preference(I, start, rf, None, 3, 200.0, 0.0, loss, margin, logp, grad)
    assert margin[0].item() == 0 and (I.rows_of(grad.cpu())[[0, 1, 9]] == 0).all()
    # no pairs at all
    loss = torch.full((1,), 7.0, device="cuda")
    grad = I.gradient()
    B.dbw_preference_loss(I.shape, 0, I.logits(), I.token_array(), torch.zeros(1, dtype=torch.int32, device="cuda"), I.scattered(rf), None,
                          0.1, 0.0, loss, I.work, None, dlogits=grad)
    assert loss.item() == 0 and (I.rows_of(grad) == 0).all()
    # offsets out of order or out of range are reported
    for bad in ([0, 5, 3], [0, 4, 11], [-1, 4, 10]):
        I.status.zero_()
        run_preference(I, bad, rf, None, 1, 0.1, 0.0, I.gradient())
        assert I.status.item() == B.ERR_INVALID
    assert base.isfinite().all()


# --------------------------------------------------------------------------- how the calls are made

def test_no_rows(B):
    shape = B.make_logits(3, 0, 100, BF16)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    e16, ei, ef = (torch.empty(0, dtype=d, device="cuda") for d in (BF16, torch.int32, F32))
    B.dbw_token_logp(shape, e16, ei, ef, work)
    B.dbw_token_logp_grad(shape, e16, ei, ef, ef, e16)
    for call in (lambda l: B.dbw_distill_loss(shape, 4, e16, ei, ef, None, l, work, dlogits=e16),
                 lambda l: B.dbw_policy_loss(shape, e16, ei, ef, ef, ef, None, 0.2, 0.2, 0.1, l, work, dlogits=e16),
                 lambda l: B.dbw_preference_loss(shape, 2, e16, ei, torch.zeros(13, dtype=torch.int32, device="cuda"), ef, None, 0.1, 0.0, l, work,
                                                 torch.empty(6, device="cuda"), dlogits=e16)):
        loss = torch.full((3,), 7.0, device="cuda")
        call(loss)
        assert torch.allclose(loss, torch.full_like(loss, math.log(2) if loss[0] != 0 else 0.0))


def _all_calls(I, seed=0):
    """Every operator on I, as closures of the gradient array; each returns what it computed besides."""
    old, rf, adv = policy_inputs(I)
    index, value, lse = teacher_of(I, min(20, I.v // 2), True, seed=seed)
    weights = torch.where(I.live, 0.5, 0.0)
    start = cut(I.total, I.n, I.t, 1, seed)
    dev = {k: v.cuda() for k, v in dict(index=index.int(), value=value, lse=lse, w=weights,
                                        start=torch.tensor(start, dtype=torch.int32)).items()}
    tokens, old, rf, adv, B = I.token_array(), I.scattered(old), I.scattered(rf), I.scattered(adv), I.B
    out = {m: torch.zeros(n, device="cuda") for m, n in dict(loss=I.n, margin=I.n, logp=I.total, lse=I.total, row=I.total).items()}
    k = index.shape[1]

    def grad(x, d):
        B.dbw_token_logp(I.shape, x, tokens, out["logp"], I.work, lse_out=out["lse"])
        B.dbw_token_logp_grad(I.shape, x, tokens, out["lse"], adv, d)
        return out["logp"]

    def distill(x, d):
        B.dbw_distill_loss(I.shape, k, x, dev["index"], dev["value"], dev["w"], out["loss"], I.work, teacher_lse=dev["lse"], dlogits=d)
        return out["loss"]

    def preference(x, d):
        B.dbw_preference_loss(I.shape, 1, x, tokens, dev["start"], rf, None, 0.1, 0.0, out["loss"], I.work, out["margin"], dlogits=d)
        return out["loss"]

    def policy(x, d):
        B.dbw_policy_loss(I.shape, x, tokens, old, rf, adv, None, 0.2, 0.28, 0.05, out["loss"], I.work, dlogits=d)
        return out["loss"]

    return {"grad": grad, "distill": distill, "preference": preference, "policy": policy}


@pytest.mark.parametrize("dtype,n,t,v", [(F32, 2, 3, 1001), (BF16, 1, 4, 20000), (F16, 1, 2, 131075), (F32, 1, 2, 150001), (BF16, 1, 2, 400000)])
def test_in_place_gives_the_same_bits(B, dtype, n, t, v):
    I = Inputs(B, dtype, n, t, v, pad=1, left=1)
    for name, call in _all_calls(I).items():
        d = I.gradient()
        first = call(I.logits(), d).clone()
        mine = I.dev.clone()
        second = call(mine, mine)
        assert torch.equal(first, second), name
        assert torch.equal(I.rows_of(mine), I.rows_of(d)), name


def test_the_same_call_gives_the_same_bits_on_another_stream(B):
    I = Inputs(B, BF16, 4, 33, 5001, left=4)
    side = torch.cuda.Stream()
    for name, call in _all_calls(I).items():
        d = I.gradient()
        first = call(I.logits(), d).clone()
        e = I.gradient()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second = call(I.logits(), e).clone()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first, second) and torch.equal(I.rows_of(d), I.rows_of(e)), name


@pytest.mark.parametrize("dtype,n,t,v", [(BF16, 2, 9, 3001), (BF16, 1, 1, 131072), (F32, 1, 2, 150001)])
def test_captured_calls_replay(B, dtype, n, t, v):
    I = Inputs(B, dtype, n, t, v)
    for name, call in _all_calls(I).items():
        d = I.gradient()
        want = call(I.logits(), d).clone()
        want_d = d.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call(I.logits(), d)
        for _ in range(3):
            d.fill_(5.0)
            got.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(I.rows_of(d), I.rows_of(want_d)), name


def test_rows_beyond_four_gigabytes(B):
    """Offsets of elements and bytes that pass 32 bits: the last rows of a long array equal the same rows in a short one."""
    v, t = 131072, 17000                                 # 4.5 GB of logits, 2.2e9 elements
    tail = Inputs(B, BF16, 1, 3, v, seed=8)
    big = torch.empty(t * v, dtype=BF16, device="cuda")
    big[(t - 3) * v:].copy_(tail.logits()[:3 * v])
    shape = B.make_logits(1, t, v, BF16)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device="cuda")
    tokens = torch.full((t,), -1, dtype=torch.int32, device="cuda")
    tokens[-3:] = tail.token_array()
    logp, lse = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    B.dbw_token_logp(shape, big, tokens, logp, work, lse_out=lse)
    want, want_lse = want_logp(tail)
    close(logp[-3:], want, tail.tol)
    grad = torch.empty_like(big)
    B.dbw_token_logp_grad(shape, big, tokens, lse, torch.ones(t, device="cuda"), grad)
    mine = tail.gradient()
    mine[:3 * v].copy_(grad[(t - 3) * v:])
    check_logp_gradient(tail, mine, torch.ones(3, dtype=torch.float64), torch.zeros(3), extra=4 * ref.U * (want_lse.abs() + 1))
    assert not grad[:(t - 3) * v].any()
