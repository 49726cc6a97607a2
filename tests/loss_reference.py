"""The losses on logits in 64 bits, from their definitions, with gradients from automatic differentiation, and how far fp32 arithmetic
may be off.

One rounding is u = 2^-24.  A log-probability is ln 2 (c x_y - M - log2 Z): c = s log2(e) is off by 2 u relative (s and the product), so a
difference of logits of at most D = 2 max |s x| by 2 u D; the argument of an exponential by u D more, log2 Z by that, by the sum's
roundings and by those of 2^x and log2 (2 u each), the products by ln 2 and the last difference by 3 u |log p|, |log p| <= D + ln V.
A thread's sum adds at most V / 64 terms one after the other, then 10 in a tree.  Together below u (8 D + V / 64 + 32); a probability's
relative error is the same.  tol() gives that number.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}    # relative, of a normal number
SUBNORMAL = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}  # absolute, below the normal numbers


def tol(x, scale):
    """Per row: bound on the error of a log-probability, and on the relative error of a probability."""
    z = (x.double() * scale).clone()
    z[torch.isinf(z)] = 0
    return U * (16 * z.abs().amax(1) + x.shape[1] / 64 + 32)


def scaled(x, scale):
    return x.double() * float(np.float32(scale))


def log_softmax(x, scale):
    return torch.log_softmax(scaled(x, scale), 1)


def token_logp(x, tokens, scale):
    return log_softmax(x, scale).gather(1, tokens.long()[:, None])[:, 0]


def distill_rows(x, index, value, scale, teacher_lse=None):
    """l_r of rows whose lists leave something; x may require a gradient."""
    lp = log_softmax(x, scale)
    there = index >= 0
    at = torch.where(there, index, 0).long()
    t = torch.where(there, scaled(value, scale), torch.tensor(-math.inf, dtype=torch.float64))
    norm = torch.logsumexp(t, 1) if teacher_lse is None else teacher_lse.double()
    log_q = t - norm[:, None]
    q = torch.exp(log_q)
    pos = q > 0
    term = torch.where(pos, q * (torch.where(pos, log_q, 0.0) - torch.where(pos, lp.gather(1, at), 0.0)), 0.0)
    out = term.sum(1)
    if teacher_lse is not None:
        inside = torch.zeros(x.shape[0], x.shape[1] + 1, dtype=torch.bool)
        inside.scatter_(1, torch.where(there, at, x.shape[1]), True)
        log_s = torch.logsumexp(torch.where(inside[:, :-1], torch.tensor(-math.inf, dtype=torch.float64), lp), 1)
        rest = (1 - q.sum(1)).clamp(min=0)
        some = rest > 0
        out = out + torch.where(some, rest * (torch.log(torch.where(some, rest, 1.0)) - torch.where(some, log_s, 0.0)), 0.0)
    return out


def policy_rows(logp, old, ref, adv, low, high, kl_coef):
    """l_r and kl_r"""
    low, high, kl_coef = (float(np.float32(v)) for v in (low, high, kl_coef))
    rho = torch.exp(logp - old.double())
    a = adv.double()
    kl = torch.zeros_like(logp)
    if ref is not None:
        d = ref.double() - logp
        kl = torch.exp(d) - d - 1
    return kl_coef * kl - torch.minimum(rho * a, rho.clamp(1 - low, 1 + high) * a), kl


def preference(logp, ref, w, start, beta, smoothing, workers, pairs):
    """loss [workers], margins [workers * pairs]; logp, ref, w of all rows (0 weight where a row takes no part)"""
    beta, smoothing = float(np.float32(beta)), float(np.float32(smoothing))
    t = w.double() * (logp - ref.double())
    h = [t[start[q]:start[q + 1]].sum() for q in range(len(start) - 1)]
    u = torch.stack([beta * (h[2 * j] - h[2 * j + 1]) for j in range(workers * pairs)])
    log_sigmoid = torch.nn.functional.logsigmoid
    l = -(1 - smoothing) * log_sigmoid(u) - smoothing * log_sigmoid(-u)
    return l.reshape(workers, pairs).mean(1), u
