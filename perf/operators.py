"""Performance cases of the losses on a language model's logits, of all simulated workers at once.

A state holds what a training or scoring program has before the call: the logits of N workers, a row of `vocab` columns for each
of a worker's `rows` token positions, with what the loss compares them with.  One pass is one operator:

  logp        log-probabilities of given tokens (scoring, and serving a token at a time)
  logp_grad   the same, then the logits' gradient from one coefficient a row (a loss of the caller's own)
  distill     distillation from a teacher's top logits: every worker's loss and the logits' gradient
  preference  paired log ratios against a reference model: losses, margins, log-probabilities and the logits' gradient
  policy      clipped policy loss with a KL term: losses, KL terms, log-probabilities and the logits' gradient

A case is a dict of plain values; listed() holds the ones that are looked at by name, draw() makes others of the same ranges.
prepare() makes the inputs, run() is one pass (the plain form, or the library's kernels where `own` is true), exact() the same
results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

OPS = ("logp", "logp_grad", "distill", "preference", "policy")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}

# left_out: rows of each worker that take no part (prompt and padding positions; their token is -1 or their weight 0)
# banned:   columns at the end of the vocabulary whose logits are -inf (a vocabulary rounded up, tokens that may not be sampled)
# pad:      elements between the end of a row and the next one's start
_BASE = {"op": "logp", "type": "bf16", "workers": 1, "rows": 1, "vocab": 1000, "pad": 0, "scale": 1.0, "left_out": 0, "banned": 0,
         "k": 0, "tail": False, "pairs": 0, "smoothing": 0.0}


def _case(name=None, **kw):
    assert set(kw) <= set(_BASE), kw
    c = {**_BASE, **kw}
    if name is not None:
        c["name"] = name
    return c


# --------------------------------------------------------------------------- the cases

def listed():
    return [
        # Serving: the log-probability of the one token just sampled, one long row.  Latency is all there is.
        _case("logp-one-token", op="logp", vocab=131072),
        # Scoring the prompts and answers of a reference model: rows are only read.
        _case("logp-score", op="logp", workers=4, rows=1024, vocab=65536, left_out=100),
        # A caller's own loss on log-probabilities, half precision, rows of an odd length one behind the other, so that hardly any
        # row starts on a boundary that a wide access likes.
        _case("logp-grad-odd-rows", op="logp_grad", type="f16", workers=3, rows=701, vocab=50001, scale=0.8, left_out=33),
        # Distillation of a small model with a short vocabulary in single precision: the smallest training step.
        _case("distill-small", op="distill", type="f32", workers=8, rows=16, vocab=1000, k=16),
        # An ordinary step of eight workers; the teacher's mass outside its top tokens is one more class.
        _case("distill-tail", op="distill", workers=8, rows=256, vocab=32000, k=64, tail=True, scale=0.5, left_out=20),
        # Long rows, more of the teacher's tokens, a vocabulary rounded up.
        _case("distill-long-rows", op="distill", workers=4, rows=1024, vocab=131072, k=128, tail=True, banned=200),
        # A few short pairs in single precision.
        _case("preference-small", op="preference", type="f32", workers=2, rows=64, vocab=32001, pairs=2, left_out=12),
        # An ordinary step: 32 pairs of ragged answers.
        _case("preference-pairs", op="preference", workers=4, rows=2048, vocab=32768, pairs=8, smoothing=0.1, left_out=300),
        # Half precision, rows of an odd length with a gap between them, one pair a worker.
        _case("preference-odd-rows", op="preference", type="f16", workers=2, rows=1500, vocab=100003, pad=13, pairs=1, left_out=151),
        # A model on bytes and a few marks, single precision.
        _case("policy-bytes", op="policy", type="f32", workers=16, rows=32, vocab=259, left_out=5),
        # An ordinary step, sampled at a temperature of 0.7.
        _case("policy-step", op="policy", workers=8, rows=512, vocab=32768, scale=1 / 0.7, left_out=77, banned=63),
        # Long rows in single precision: a row is half a megabyte.
        _case("policy-long-rows-f32", op="policy", type="f32", workers=2, rows=1024, vocab=131072, left_out=128),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(OPS)
    kind = rng.choice(("f32", "bf16", "bf16", "f16"))
    vocab = _log_uniform(rng, 64, 131072)
    vocab = vocab | 1 if rng.random() < 0.5 else max(80, vocab // 80 * 80)      # rows of odd lengths, rows on 16-byte boundaries
    workers = _log_uniform(rng, 1, 32)
    budget = 1 << 30                                     # bytes of logits, those of the largest listed case
    most = max(2, min(2500, budget // (workers * (vocab + 16) * SIZE[kind])))
    rows = _log_uniform(rng, 1 if op.startswith("logp") else 2, most)
    c = _case(op=op, type=kind, workers=workers, rows=rows, vocab=vocab, pad=rng.choice((0, 0, 0, 1, 8, 13)),
              scale=rng.choice((1.0, 1.0, 0.5, 1.25)), left_out=rng.randint(0, rows // 3), banned=rng.choice((0, 0, vocab // 50)))
    if op == "distill":
        c["k"] = _log_uniform(rng, 1, min(256, vocab // 4))
        c["tail"] = rng.random() < 0.5
    if op == "preference":
        c["pairs"] = _log_uniform(rng, 1, max(1, min(16, rows // 2)))
        c["smoothing"] = rng.choice((0.0, 0.1))
    return c


# --------------------------------------------------------------------------- inputs

BETA, CLIP_LOW, CLIP_HIGH, KL_COEF = 0.1, 0.2, 0.28, 0.05


def _logp_of(logits, tokens, scale):
    """Log-probabilities for making the other models' figures, a piece of the rows at a time."""
    out = torch.empty(tokens.numel(), device=logits.device)
    step = max(1, (1 << 26) // logits.shape[1])
    for a in range(0, out.numel(), step):
        z = logits[a:a + step].float() * scale
        y = tokens[a:a + step].clamp(min=0).long()
        m = z.amax(1)
        out[a:a + step] = z.gather(1, y[:, None])[:, 0] - m - torch.log(torch.exp(z - m[:, None]).sum(1))
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n, t, v = case["workers"], case["rows"], case["vocab"]
    rows, ld, usable = n * t, v + case["pad"], v - case["banned"]
    kind = TYPES[case["type"]]

    def rand(*size):
        return torch.rand(*size, device=dev, generator=g)

    def normal(*size):
        return torch.randn(*size, device=dev, generator=g)

    # a trained model's rows: a broad floor of unlikely tokens, a few likely ones, the given token often among them
    flat = torch.empty(rows, ld, device=dev, dtype=kind).normal_(generator=g)
    flat *= 2.0
    logits = flat[:, :v]
    if case["banned"]:
        logits[:, usable:] = -math.inf
    tokens = torch.randint(0, usable, (rows,), device=dev, generator=g)
    peak = (normal(rows) * 4 + 8).to(kind)
    logits[torch.arange(rows, device=dev), tokens] = peak
    other = torch.randint(0, usable, (rows, 4), device=dev, generator=g)
    logits.scatter_(1, other, (normal(rows, 4) * 3 + 6).to(kind))

    s = {"case": dict(case), "flat": flat, "scale": case["scale"]}
    # the rows that take part: left_out of each worker's do not
    order = rand(n, t).argsort(1)
    live = torch.ones(n, t, dtype=torch.bool, device=dev)
    live.scatter_(1, order[:, :case["left_out"]], False)
    live = live.reshape(rows)
    weights = torch.where(live, 1.0 / (t - case["left_out"]), 0.0).to(torch.float32)
    op = case["op"]
    if op != "distill":
        # a row without a token is one that takes no part
        s["tokens"] = torch.where(live, tokens, -1).to(torch.int32)
    if op == "logp_grad":
        s["coef"] = normal(rows) * weights * live
    elif op == "distill":
        k = case["k"]
        # The teacher agrees with the student on some of the likely tokens; its indices are distinct, best first, and short
        # lists end in -1.
        pick = torch.cat([tokens[:, None], other], 1)
        some = torch.randint(0, usable, (rows, 4 * k + 8), device=dev, generator=g)
        cand = torch.cat([pick, some], 1).sort(1).values
        fresh = torch.ones_like(cand, dtype=torch.bool)
        fresh[:, 1:] = cand[:, 1:] != cand[:, :-1]
        key = torch.where(fresh, rand(rows, cand.shape[1]), -1.0) + torch.where((cand == tokens[:, None]) & fresh, 1.0, 0.0)
        top = key.topk(k, 1)
        index = torch.where(top.values >= 0, cand.gather(1, top.indices), -1)
        value = (normal(rows, k) * 3 + 2).sort(1, descending=True).values
        if k > 2:
            short = rand(rows) < 0.1
            index[:, k - k // 3:] = torch.where(short[:, None], -1, index[:, k - k // 3:])
        s["index"] = index.to(torch.int32)
        s["value"] = value
        if case["tail"]:
            z = torch.where(index >= 0, value * case["scale"], -math.inf)
            m = z.amax(1)
            top_mass = torch.log(torch.exp(z - m[:, None]).sum(1)) + m
            s["teacher_lse"] = top_mass - torch.log(1 - (rand(rows) * 0.3 + 0.002))     # 0.2 to 30 % of the mass lies outside
        s["weights"] = weights
    elif op in ("preference", "policy"):
        now = _logp_of(logits, s["tokens"], case["scale"])
        s["weights"] = weights if op == "policy" else live.to(torch.float32)
        s["ref_logp"] = torch.where(live, now + normal(rows) * 0.2, math.nan)            # nobody filled in the rest
        if op == "policy":
            # Ratios to the sampling model around one, a good part of them clipped.  The gradient jumps where a ratio meets a
            # bound, where both branches are right: no ratio lies within 1e-3 of one.
            step = normal(rows) * 0.2
            for bound in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
                step = torch.where((step - bound).abs() < 1e-3, bound + 2e-3, step)
            s["old_logp"] = torch.where(live, now - step, math.nan)
            s["advantage"] = normal(rows)
        else:
            cuts = torch.sort(torch.randint(0, t + 1, (n, 2 * case["pairs"] - 1), device=dev, generator=g), 1).values
            start = torch.cat([torch.zeros(n, 1, dtype=cuts.dtype, device=dev), cuts], 1) + t * torch.arange(n, device=dev)[:, None]
            s["start"] = torch.cat([start.reshape(-1), torch.tensor([rows], device=dev)]).to(torch.int32)
    if own:
        from paper_2102_06280_amd import binding as B
        number = {"f32": B.TYPE_F32, "bf16": B.TYPE_BF16, "f16": B.TYPE_F16}[case["type"]]
        s["shape"] = shape = B.make_logits(n, t, v, number, ld=ld, ld_grad=v, scale=case["scale"])
        s["work"] = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8, device=dev)
        s["logp"] = torch.empty(rows, device=dev)
        if op == "logp_grad":
            s["lse"] = torch.empty(rows, device=dev)
        if op != "logp":
            s["grad"] = torch.empty(rows, v, device=dev, dtype=kind)
        s["loss"] = torch.empty(n, device=dev)
        s["kl"] = torch.empty(n, device=dev)
        s["margin"] = torch.empty(n * max(case["pairs"], 1), device=dev)
    return s


# --------------------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2102_06280_amd import binding as B
    op = s["case"]["op"]
    if op == "logp":
        B.dbw_token_logp(s["shape"], s["flat"], s["tokens"], s["logp"], s["work"])
        return {"logp": s["logp"]}
    if op == "logp_grad":
        B.dbw_token_logp(s["shape"], s["flat"], s["tokens"], s["logp"], s["work"], lse_out=s["lse"])
        B.dbw_token_logp_grad(s["shape"], s["flat"], s["tokens"], s["lse"], s["coef"], s["grad"])
        return {"logp": s["logp"], "grad": s["grad"]}
    if op == "distill":
        B.dbw_distill_loss(s["shape"], s["case"]["k"], s["flat"], s["index"], s["value"], s["weights"], s["loss"], s["work"],
                           teacher_lse=s.get("teacher_lse"), dlogits=s["grad"])
        return {"loss": s["loss"], "grad": s["grad"]}
    if op == "preference":
        B.dbw_preference_loss(s["shape"], s["case"]["pairs"], s["flat"], s["tokens"], s["start"], s["ref_logp"], s["weights"], BETA,
                              s["case"]["smoothing"], s["loss"], s["work"], margin_out=s["margin"], logp_out=s["logp"],
                              dlogits=s["grad"])
        return {"loss": s["loss"], "margin": s["margin"], "logp": s["logp"], "grad": s["grad"]}
    B.dbw_policy_loss(s["shape"], s["flat"], s["tokens"], s["old_logp"], s["ref_logp"], s["advantage"], s["weights"], CLIP_LOW,
                      CLIP_HIGH, KL_COEF, s["loss"], s["work"], kl_out=s["kl"], logp_out=s["logp"], dlogits=s["grad"])
    return {"loss": s["loss"], "kl": s["kl"], "logp": s["logp"], "grad": s["grad"]}


def _run_plain(s):
    case = s["case"]
    n, v, op, scale = case["workers"], case["vocab"], case["op"], s["scale"]
    z = s["flat"][:, :v].float() * scale
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    if op == "distill":
        index, w = s["index"].long(), s["weights"]
        there, at = index >= 0, index.clamp(min=0)
        teacher = torch.where(there, s["value"] * scale, -math.inf)
        if case["tail"]:
            norm = s["teacher_lse"][:, None]
        else:
            top = teacher.amax(1, keepdim=True)
            norm = top + torch.log(torch.exp(teacher - top).sum(1, keepdim=True))
        q = torch.exp(teacher - norm)
        logp = z.gather(1, at) - m - torch.log(total)
        row = torch.where(q > 0, q * (teacher - norm - logp), 0.0).sum(1)
        p = e / total
        mine = torch.where(there, p.gather(1, at) - q, 0.0)
        if case["tail"]:
            rest = (1 - q.sum(1)).clamp(min=0)
            outside = e.clone()
            outside.scatter_(1, torch.where(there, at, at[:, :1]), 0.0)      # the first index is always there
            mass = outside.sum(1) / total[:, 0]
            row = row + rest * (torch.log(rest) - torch.log(mass))
            grad = p * (1 - rest / mass)[:, None]
        else:
            grad = p
        grad.scatter_(1, torch.where(there, at, at[:, :1]), torch.where(there, mine, mine[:, :1]))
        on = w > 0
        grad = torch.where(on[:, None], grad * (scale * w)[:, None], 0.0)
        loss = torch.where(on, w * row, 0.0).reshape(n, -1).sum(1)
        return {"loss": loss, "grad": grad.to(s["flat"].dtype)}

    tokens = s["tokens"].long()
    live, y = tokens >= 0, tokens.clamp(min=0)[:, None]
    logp = torch.where(live, (z.gather(1, y) - m - torch.log(total))[:, 0], 0.0)
    if op == "logp":
        return {"logp": logp}
    out = {}
    if op == "logp_grad":
        coef = s["coef"]
    elif op == "preference":
        w, start = s["weights"], s["start"].long()
        ratio = torch.where(live, w * (logp - s["ref_logp"]), 0.0)
        position = torch.arange(logp.numel(), device=logp.device)
        seq = (position[:, None] >= start[None, 1:]).sum(1)                  # the sequence that a row lies in
        member = seq[None, :] == torch.arange(2 * n * case["pairs"], device=logp.device)[:, None]
        sums = torch.where(member, ratio[None, :], 0.0).sum(1).reshape(-1, 2)
        u = BETA * (sums[:, 0] - sums[:, 1])
        a = case["smoothing"]
        softplus = torch.clamp(u, min=0) + torch.log1p(torch.exp(-u.abs()))  # log(1 + exp(u))
        out["loss"] = (softplus - (1 - a) * u).reshape(n, -1).sum(1) / case["pairs"]
        out["margin"] = u
        slope = (1 / (1 + torch.exp(-u)) - (1 - a)) * (BETA / case["pairs"])
        coef = torch.where(live, w * torch.stack([slope, -slope], 1).reshape(-1)[seq], 0.0)
    else:
        w, adv = s["weights"], s["advantage"]
        rho = torch.exp(logp - s["old_logp"])
        d = s["ref_logp"] - logp
        kl = torch.exp(d) - d - 1
        clipped = torch.clamp(rho, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
        row = -torch.minimum(rho * adv, clipped) + KL_COEF * kl
        out["loss"] = torch.where(live, w * row, 0.0).reshape(n, -1).sum(1)
        out["kl"] = torch.where(live, w * kl, 0.0).reshape(n, -1).sum(1)
        slope = torch.where(rho * adv <= clipped, -adv * rho, 0.0) + KL_COEF * (1 - torch.exp(d))
        coef = torch.where(live, w * slope, 0.0)
    coef = torch.where(live, coef, 0.0) * scale
    grad = e * (-coef[:, None] / total)
    grad.scatter_add_(1, y, coef[:, None])
    out["logp"] = logp
    out["grad"] = torch.where((coef != 0)[:, None], grad, 0.0).to(s["flat"].dtype)
    return out


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = SIZE[case["type"]]
    rows = case["workers"] * case["rows"]
    live = case["workers"] * (case["rows"] - case["left_out"])
    v, op = case["vocab"], case["op"]
    bytes_ = live * v * size + rows * 4                     # the logits, the tokens or weights
    flops = live * v * 4                                    # scale and subtract, exp, add
    if op != "logp":
        bytes_ += rows * v * size                           # the gradient
        flops += live * v * 4
    if op != "distill":
        bytes_ += rows * 4                                  # log-probabilities
    if op == "logp_grad":
        bytes_ += rows * 4
    elif op == "distill":
        bytes_ += live * case["k"] * 8 + (live * 4 if case["tail"] else 0) + case["workers"] * 4
    elif op == "preference":
        bytes_ += rows * 8 + case["workers"] * (16 * case["pairs"] + 4)
    elif op == "policy":
        bytes_ += rows * 4 + live * 12 + case["workers"] * 8
    return {"bytes": bytes_, "flops": flops}


# --------------------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    """From the definitions, in 64 bits: log softmax of a row, its loss, and the loss's derivative."""
    s = prepare(case, seed)
    n, t, v, op, scale = case["workers"], case["rows"], case["vocab"], case["op"], case["scale"]
    rows = n * t
    dev = s["flat"].device
    logp = torch.zeros(rows, dtype=torch.float64, device=dev)
    grad = torch.zeros(rows, v, dtype=torch.float64, device=dev) if op != "logp" else None
    loss_row = torch.zeros(rows, dtype=torch.float64, device=dev)
    on = (s["weights"] != 0) if op == "distill" else (s["tokens"] >= 0)
    chosen = torch.nonzero(on)[:, 0]
    step = max(1, (1 << 25) // v)
    pieces = [chosen[a:a + step] for a in range(0, chosen.numel(), step)]

    def log_probabilities(r):
        return torch.log_softmax(s["flat"][r, :v].double() * scale, 1)

    if op == "distill":
        for r in pieces:
            lp = log_probabilities(r)
            index, w = s["index"][r].long(), s["weights"][r].double()
            for_each = torch.zeros(r.numel(), v + 1, dtype=torch.float64, device=dev)         # column v takes what is absent
            teacher = s["value"][r].double() * scale
            teacher = teacher.masked_fill(index < 0, -math.inf)
            norm = s["teacher_lse"][r].double() if case["tail"] else torch.logsumexp(teacher, 1)
            for_each.scatter_(1, torch.where(index < 0, v, index), torch.exp(teacher - norm[:, None]))
            q = for_each[:, :v]
            inside = torch.zeros(r.numel(), v + 1, dtype=torch.bool, device=dev)
            inside.scatter_(1, torch.where(index < 0, v, index), True)
            inside = inside[:, :v]
            terms = torch.where(q > 0, q * (torch.log(q) - lp), 0.0).sum(1)
            p = torch.exp(lp)
            d = p - q
            if case["tail"]:
                rest = 1 - q.sum(1)
                mass = torch.where(inside, 0.0, p).sum(1)
                terms = terms + rest * torch.log(rest / mass)
                d = torch.where(inside, d, p - (rest / mass)[:, None] * p)
            loss_row[r] = w * terms
            grad[r] = d * (scale * w)[:, None]
        return {"loss": loss_row.reshape(n, t).sum(1), "grad": grad}

    for r in pieces:
        logp[r] = log_probabilities(r).gather(1, s["tokens"][r].long()[:, None])[:, 0]
    if op == "logp":
        return {"logp": logp}
    out = {}
    slope = torch.zeros_like(logp)
    if op == "logp_grad":
        slope[chosen] = s["coef"][chosen].double()
    elif op == "preference":
        start = s["start"].tolist()
        w = s["weights"].double()
        ratio = torch.zeros_like(logp)
        ratio[chosen] = w[chosen] * (logp[chosen] - s["ref_logp"][chosen].double())
        pairs = case["pairs"]
        losses, margins = [], []
        for pair in range(n * pairs):
            c, r = slice(start[2 * pair], start[2 * pair + 1]), slice(start[2 * pair + 1], start[2 * pair + 2])
            u = BETA * float(ratio[c].sum() - ratio[r].sum())
            yes, no = 1 / (1 + math.exp(-u)), 1 / (1 + math.exp(u))
            losses.append(-(1 - case["smoothing"]) * math.log(yes) - case["smoothing"] * math.log(no))
            margins.append(u)
            by = BETA / pairs * (case["smoothing"] * yes - (1 - case["smoothing"]) * no)
            slope[c], slope[r] = by * w[c], -by * w[r]
        out["loss"] = torch.tensor(losses, dtype=torch.float64, device=dev).reshape(n, pairs).mean(1)
        out["margin"] = torch.tensor(margins, dtype=torch.float64, device=dev)
        slope = torch.where(on, slope, 0.0)
    else:
        w, a = s["weights"][chosen].double(), s["advantage"][chosen].double()
        rho = torch.exp(logp[chosen] - s["old_logp"][chosen].double())
        gone = torch.exp(s["ref_logp"][chosen].double() - logp[chosen])
        kl = gone - torch.log(gone) - 1
        bounded = rho.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
        loss_row[chosen] = w * (KL_COEF * kl - torch.minimum(rho * a, bounded * a))
        out["loss"] = loss_row.reshape(n, t).sum(1)
        kl_row = torch.zeros_like(logp)
        kl_row[chosen] = w * kl
        out["kl"] = kl_row.reshape(n, t).sum(1)
        free = torch.where(a > 0, rho <= 1 + CLIP_HIGH, rho >= 1 - CLIP_LOW)
        slope[chosen] = w * (KL_COEF * (1 - gone) - torch.where(free, rho * a, 0.0))
    for r in pieces:
        d = -torch.exp(log_probabilities(r))
        d.scatter_add_(1, s["tokens"][r].long()[:, None], torch.ones(r.numel(), 1, dtype=torch.float64, device=dev))
        grad[r] = d * (scale * slope[r])[:, None]
    out["logp"], out["grad"] = logp, grad
    return out
