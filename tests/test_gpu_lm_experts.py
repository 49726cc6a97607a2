"""A language model with a norm and experts between its products, through the library's layers: its gradients against autograd in 64 bits, and the study with
such models."""
import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu


def reference(models, context, dlogits):
    """Gradients of (logits * dlogits).sum() in 64 bits, by autograd, of the parameters' rows, and what the bounds below need."""
    from paper_2102_06280_amd import lm_study as L
    rows = models.rows.detach().cpu().double().requires_grad_()
    m = L.ExpertModels(rows, models.experts)
    context, dlogits = context.cpu(), dlogits.cpu().double()
    n = torch.arange(context.shape[0])[:, None]
    hidden = torch.tanh(m.first[n, context[..., 0]] + m.second[n, context[..., 1]])
    hidden.retain_grad()
    mu = hidden.mean(-1, keepdim=True)
    rho = 1 / torch.sqrt((hidden - mu).square().mean(-1, keepdim=True) + 1e-5)
    plain = (hidden - mu) * rho
    unit = plain * m.norm_weight[:, None] + m.norm_bias[:, None]
    unit.retain_grad()
    top = torch.einsum("ntw,new->nte", unit, m.router).topk(L.CHOSEN, -1)
    share = torch.softmax(top.values, -1)
    z = torch.einsum("ntjvw,ntw->ntjv", m.weight[n[..., None], top.indices], unit) + m.shift[n[..., None], top.indices]
    z.retain_grad()
    out = hidden + (share[..., None] * z).sum(2)
    logits = torch.einsum("ntw,nvw->ntv", out, m.out) + m.bias[:, None]
    (logits * dlogits).sum().backward()
    return logits.detach(), rows.grad, {"hidden": hidden.detach(), "unit": unit.detach(), "dunit": unit.grad, "dz": z.grad, "choice": top.indices, "rho": rho.detach(),
                                        "plain": plain.detach(), "top": top.values.detach()}


def test_gradients_of_a_model_with_experts():
    """What passes through 8 bits is off by what they round, 2^-4 of a value at most (or 2^-10 of its block's power of two, less than 2^-17 of the largest value); the
    rest by fp32 arithmetic, of which 1e-5 of the gradient's size is much more than the few dozen roundings on the way."""
    from paper_2102_06280_amd import lm_study as L
    workers, tokens, experts, W = 3, 40, 5, L.WIDTH
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = torch.randn(workers, L.ExpertModels.size(experts) + 9, device="cuda", generator=g) * 0.4
    models = L.ExpertModels(rows, experts)
    models.norm_weight += 1
    context = torch.randint(0, L.VOCAB, (workers, tokens, 2), device="cuda", generator=g)
    dlogits = torch.randn(workers, tokens, L.VOCAB, device="cuda", generator=g) * 0.01
    logits, state = models.forward(context)
    grads = torch.full_like(rows, 7.0)
    models.backward(context, state, dlogits, grads)
    want_logits, want, seen = reference(models, context, dlogits)
    assert torch.equal(state["choice"].cpu(), seen["choice"])
    assert (logits.cpu().double() - want_logits).abs().max() < 1e-5 * want_logits.abs().max()
    got, mine, theirs = grads.cpu().double(), L.ExpertModels(grads.cpu().double(), experts), L.ExpertModels(want, experts)
    assert (got[:, -9:] == 7).all()
    near = lambda a, b, bound=0.0: ((a - b).abs() <= bound + 1e-5 * b.abs().max()).all()
    # not through 8 bits: the output's, and the router's
    assert near(mine.out, theirs.out) and near(mine.bias, theirs.bias) and near(mine.router, theirs.router)
    assert near(mine.shift, theirs.shift) and near(mine.norm_bias, theirs.norm_bias)
    # an expert's weights: dz u, with u off by 2^-4 |u| + 2^-17 max |u|
    off = lambda v: 2.0 ** -4 * v.abs() + 2.0 ** -17 * v.abs().amax(-1, keepdim=True)
    bound = torch.zeros_like(theirs.weight)
    for i in range(workers):
        for e in range(experts):
            for t, j in (seen["choice"][i] == e).nonzero().tolist():
                bound[i, e] += seen["dz"][i, t, j].abs()[:, None] * off(seen["unit"][i, t])[None]
    assert near(mine.weight, theirs.weight, bound)
    assert ((mine.weight - theirs.weight).abs() > 1e-5 * theirs.weight.abs().max()).any()      # (they do pass through 8 bits)
    # the norm: (h - mu) rho, with h off by off(h); d = rho off(h)
    d = seen["rho"] * off(seen["hidden"])
    assert near(mine.norm_weight, theirs.norm_weight, (seen["dunit"].abs() * d).sum(1))
    gw = (seen["dunit"] * models.norm_weight.cpu().double()[:, None]).abs()
    u = seen["plain"].abs()
    dh = seen["rho"] * (d * (gw * u).mean(-1, keepdim=True) + (u + d) * (gw * d).mean(-1, keepdim=True))
    dh = dh * (1 - seen["hidden"] ** 2)
    for k, name in enumerate(("first", "second")):
        which = torch.nn.functional.one_hot(context[..., k].cpu(), L.VOCAB).double()
        assert near(getattr(mine, name), getattr(theirs, name), which.transpose(1, 2) @ dh), name


def test_the_study_runs_with_experts_and_repeats():
    from paper_2102_06280_amd import binding as B
    from paper_2102_06280_amd import lm_study
    a = lm_study.run(workers=4, rounds=3, experts=4)
    assert a["status"] == B.OK and all(np.isfinite(a[k]).all() for k in a if k != "status")
    assert a["params"].shape == (4, lm_study.ExpertModels.size(4))
    b = lm_study.run(workers=4, rounds=3, experts=4)
    assert np.array_equal(a["params"], b["params"])
