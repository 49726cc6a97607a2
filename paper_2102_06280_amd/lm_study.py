"""Small language models of N workers trained through the library's losses on logits and its rounds.

Three stages, one after the other, on synthetic tokens: distillation from a fixed teacher's top logits, a preference
loss on pairs of answers, and a clipped policy loss with a KL term on sampled tokens.  Every round is the same: the
workers' logits, a loss of dbw_losses.h with the logits' gradient, from that the models' gradients, the selection of
neighbours from the round's response times, and dbw_round with the gradients as ext_grads.  Losses, gradients of the
logits, selection, averaging and local step are the library's; the model (a hidden layer on the last two tokens) and
its backward pass are the caller's, a few products of torch in fp32.  With --experts there is a layer more between the hidden
one and the output: a norm, and two of so many experts for every token; the norm, the way of the tokens to their experts and
back and the gradients of all that are the library's (dbw_layers.h), and what the backward pass needs is kept in 8 bits.

    python -m paper_2102_06280_amd.lm_study [--workers 6] [--rounds 40] [--experts 0]
"""
from __future__ import annotations

import argparse
import json

import numpy as np
import torch

from . import binding as B
from . import inputs

VOCAB, WIDTH = 260, 16                 # bytes and four marks
ROWS, PAIRS, TOP = 64, 4, 16           # token positions and pairs of each worker's batch, the teacher's tokens
SCALE, BETA, CLIP_LOW, CLIP_HIGH, KL_COEF = 1.0, 1.0, 0.2, 0.28, 0.02
D = 3 * VOCAB * WIDTH + VOCAB


class Models:
    """N models with their parameters in the library's rows [N, ld]: two embeddings, the output weight and its bias."""

    def __init__(self, rows: torch.Tensor):
        n = rows.shape[0]
        part = VOCAB * WIDTH
        self.first, self.second, self.out = (rows[:, k * part:(k + 1) * part].view(n, VOCAB, WIDTH) for k in range(3))
        self.bias = rows[:, 3 * part:D]

    def forward(self, context):
        """context [N, T, 2] -> logits [N, T, VOCAB] and what the backward pass needs."""
        n = torch.arange(context.shape[0], device=context.device)[:, None]
        hidden = torch.tanh(self.first[n, context[..., 0]] + self.second[n, context[..., 1]])
        return torch.bmm(hidden, self.out.transpose(1, 2).contiguous()) + self.bias[:, None], hidden

    def backward(self, context, hidden, dlogits, grads: torch.Tensor):
        """Gradients of the parameters into rows [N, ld]; products only, so that no sum depends on an order."""
        g = Models(grads)
        g.out.copy_(torch.bmm(dlogits.transpose(1, 2).contiguous(), hidden))
        g.bias.copy_(dlogits.sum(1))
        self._into_embeddings(context, torch.bmm(dlogits, self.out.contiguous()) * (1 - hidden * hidden), g)

    @staticmethod
    def _into_embeddings(context, dhidden, g):
        for k, into in enumerate((g.first, g.second)):
            which = torch.nn.functional.one_hot(context[..., k], VOCAB).float()
            into.copy_(torch.bmm(which.transpose(1, 2).contiguous(), dhidden))


CHOSEN = 2                             # experts of a token


class ExpertModels(Models):
    """Models with a layer of experts: h' = h + sum over the token's experts of w_e (W_e u + b_e), u the norm of h, w the softmax of the chosen
    experts' router logits R u.  Parameters behind those of Models: the norm's weight and bias, R, all W_e, all b_e."""

    def __init__(self, rows: torch.Tensor, experts: int):
        super().__init__(rows)
        self.rows, self.experts, n = rows, experts, rows.shape[0]
        sizes = [WIDTH, WIDTH, experts * WIDTH, experts * WIDTH * WIDTH, experts * WIDTH]
        self.at = [D + sum(sizes[:i]) for i in range(len(sizes))]
        part = [rows[:, a:a + size] for a, size in zip(self.at, sizes)]
        self.norm_weight, self.norm_bias = part[:2]
        self.router, self.weight, self.shift = part[2].view(n, experts, WIDTH), part[3].view(n, experts, WIDTH, WIDTH), part[4].view(n, experts, WIDTH)

    @staticmethod
    def size(experts: int) -> int:
        return D + 2 * WIDTH + experts * WIDTH * (WIDTH + 2)

    def _chosen(self, of, state):
        """The sorted rows' experts' share of a parameter [N, E, ...]."""
        return of[state["worker"], state["expert"]]

    def forward(self, context):
        n = torch.arange(context.shape[0], device=context.device)[:, None]
        tokens = context.shape[0] * context.shape[1]
        hidden = torch.tanh(self.first[n, context[..., 0]] + self.second[n, context[..., 1]])
        shape = B.make_rows(*context.shape[:2], WIDTH, B.TYPE_F32)
        routing = B.make_routing(*context.shape[:2], CHOSEN, self.experts)
        empty = lambda rows, width=WIDTH, dtype=torch.float32: torch.empty(rows, width, device=context.device, dtype=dtype)
        whole = lambda count: torch.empty(count, device=context.device, dtype=torch.int32)
        memory = lambda size: torch.empty(size, device=context.device, dtype=torch.uint8)
        s = {"shape": shape, "routing": routing, "hidden": hidden, "stats": empty(tokens, 2), "kept_hidden": memory(B.dbw_checkpoint_bytes(shape)),
             "kept_unit": memory(B.dbw_checkpoint_bytes(shape)), "start": whole(context.shape[0] * (self.experts + 1)),
             "place": whole(tokens * CHOSEN), "source": whole(tokens * CHOSEN)}
        unit, sorted_rows, out = empty(tokens), empty(tokens * CHOSEN), empty(tokens)
        B.dbw_layer_norm(shape, hidden, self.rows, unit, weight_at=self.at[0], bias_at=self.at[1], stats_out=s["stats"], checkpoint=s["kept_hidden"])
        B.dbw_checkpoint_store(shape, unit, s["kept_unit"])
        unit = unit.view(hidden.shape)
        top = torch.bmm(unit, self.router.transpose(1, 2).contiguous()).topk(CHOSEN, -1)
        s["unit"], s["choice"], s["share"] = unit, top.indices, torch.softmax(top.values, -1)
        B.dbw_expert_sort(routing, top.indices.int(), s["start"], s["place"], s["source"], memory(B.dbw_expert_work_bytes(routing)))
        B.dbw_expert_gather(routing, shape, unit, s["place"], sorted_rows)
        slot = s["source"].long()
        s["worker"], s["expert"] = slot // (context.shape[1] * CHOSEN), top.indices.reshape(-1)[slot]
        s["result"] = torch.bmm(self._chosen(self.weight, s), sorted_rows[..., None])[..., 0] + self._chosen(self.shift, s)
        B.dbw_expert_combine(routing, shape, s["result"], s["place"], out, weights=s["share"])
        s["out"] = hidden + out.view(hidden.shape)
        return torch.bmm(s["out"], self.out.transpose(1, 2).contiguous()) + self.bias[:, None], s

    def backward(self, context, s, dlogits, grads: torch.Tensor):
        g = ExpertModels(grads, self.experts)
        shape, routing, hidden = s["shape"], s["routing"], s["hidden"]
        memory = lambda size: torch.empty(size, device=context.device, dtype=torch.uint8)
        g.out.copy_(torch.bmm(dlogits.transpose(1, 2).contiguous(), s["out"]))
        g.bias.copy_(dlogits.sum(1))
        dout = torch.bmm(dlogits, self.out.contiguous())
        dresult, dshare = torch.empty_like(s["result"]), torch.empty_like(s["share"])
        B.dbw_expert_combine_grad(routing, shape, dout, s["result"], s["place"], dresult, weights=s["share"], dweights=dshare)
        linear = B.make_linear(routing.workers, routing.tokens * CHOSEN, WIDTH, WIDTH, B.TYPE_F32, experts=self.experts, tokens=routing.tokens, k=CHOSEN)
        B.dbw_checkpoint_weight_grad(linear, dresult, s["kept_unit"], grads, memory(B.dbw_checkpoint_weight_grad_work_bytes(linear)), self.at[3],
                                     bias_at=self.at[4], start=s["start"], source=s["source"])
        dsorted = torch.bmm(dresult[:, None], self._chosen(self.weight, s))[:, 0]
        dunit = torch.empty_like(hidden)
        B.dbw_expert_combine(routing, shape, dsorted, s["place"], dunit)
        dchosen = s["share"] * (dshare - (s["share"] * dshare).sum(-1, keepdim=True))
        drouter = torch.zeros(*hidden.shape[:2], self.experts, device=hidden.device).scatter_(-1, s["choice"], dchosen)
        g.router.copy_(torch.bmm(drouter.transpose(1, 2).contiguous(), s["unit"]))
        dunit += torch.bmm(drouter, self.router.contiguous())
        dhidden = torch.empty_like(hidden)
        B.dbw_layer_norm_grad(shape, dunit, None, s["stats"], self.rows, dhidden, grads, memory(B.dbw_layer_norm_work_bytes(shape)),
                              weight_at=self.at[0], bias_at=self.at[1], checkpoint=s["kept_hidden"])
        self._into_embeddings(context, (dout + dhidden) * (1 - hidden * hidden), g)


class Study:
    def __init__(self, workers: int, seed: int = 1, experts: int = 0):
        self.n = workers
        self.models = (lambda rows: ExpertModels(rows, experts)) if experts else Models
        d = ExpertModels.size(experts) if experts else D
        self.d, self.ld = d, inputs.pad_ld(d)
        g = np.random.default_rng(seed)
        self.times = g
        rowptr, colidx = inputs.graph_ring(workers) if workers > 2 else inputs.graph_complete(workers)
        self.backups = torch.from_numpy((np.diff(rowptr) > 1).astype(np.int32)).cuda()       # one backup worker where there are two
        self.h = B.dbw_create(rowptr, colidx, workers, d, ld=self.ld)
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        draw = lambda rows, spread: torch.randn(rows, self.ld, device="cuda", generator=self.gen) * spread
        self.teacher_rows = draw(1, 1.5).expand(workers, -1).contiguous()
        self.teacher = Models(self.teacher_rows)
        self.x = [draw(workers, 0.3), torch.zeros(workers, self.ld, device="cuda")]
        if experts:
            start = self.models(self.x[0])
            start.norm_weight.fill_(1.0)
            start.norm_bias.zero_()
        self.grads = torch.zeros(workers, self.ld, device="cuda")
        # what the losses need: a shape, scratch memory, outputs
        self.shape = B.make_logits(workers, ROWS, VOCAB, B.TYPE_F32, scale=SCALE)
        self.work = torch.empty(B.dbw_loss_work_bytes(self.shape), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.diverged = torch.zeros((), dtype=torch.int64, device="cuda")      # tokens sampled from no distribution
        self.dlogits = torch.empty(workers, ROWS, VOCAB, device="cuda")
        self.loss = torch.empty(workers, device="cuda")

    def close(self):
        B.dbw_destroy(self.h)

    def contexts(self):
        return torch.randint(0, VOCAB, (self.n, ROWS, 2), device="cuda", generator=self.gen)

    def sample(self, logits):
        # (of a model that has diverged any token is as good as another, and is counted: multinomial ends the process where a probability is none)
        p = torch.softmax(logits * SCALE, -1).reshape(-1, VOCAB)
        none = torch.isnan(p).any(-1)
        self.diverged += none.sum()
        p.masked_fill_(none[:, None], 1.0)
        return torch.multinomial(p, 1, generator=self.gen)[:, 0].int()

    def logp(self, models, context, tokens):
        out = torch.empty(self.n * ROWS, device="cuda")
        B.dbw_token_logp(self.shape, models.forward(context)[0], tokens, out, self.work, status_out=self.status)
        return out

    def round(self, context, hidden, lr):
        """From the logits' gradient to the parameters after the round."""
        self.models(self.x[0]).backward(context, hidden, self.dlogits, self.grads)
        t = torch.from_numpy(self.times.standard_exponential(self.n).astype(np.float32)).cuda()
        B.dbw_select(self.h, t, self.backups)
        B.dbw_round(self.h, self.x[0], self.x[1], lr, ext_grads=self.grads)
        self.x.reverse()

    def distill(self, lr):
        context = self.contexts()
        logits, hidden = self.models(self.x[0]).forward(context)
        of_teacher = self.teacher.forward(context)[0]
        top = of_teacher.topk(TOP, -1)
        B.dbw_distill_loss(self.shape, TOP, logits, top.indices.int(), top.values.contiguous(), None, self.loss, self.work,
                           teacher_lse=torch.logsumexp(of_teacher * SCALE, -1), dlogits=self.dlogits, status_out=self.status)
        self.round(context, hidden, lr)
        return self.loss.clone()

    def preference(self, reference, lr):
        """Answers of ROWS / (2 PAIRS) tokens: the teacher's are preferred to random ones."""
        length = ROWS // (2 * PAIRS)
        context = self.contexts()
        good = self.sample(self.teacher.forward(context)[0])
        bad = torch.randint(0, VOCAB, good.shape, device="cuda", generator=self.gen).int()
        odd = (torch.arange(self.n * ROWS, device="cuda") // length) % 2 == 1
        tokens = torch.where(odd, bad, good)
        start = torch.arange(0, self.n * ROWS + 1, length, device="cuda").int()
        logits, hidden = self.models(self.x[0]).forward(context)
        margin = torch.empty(self.n * PAIRS, device="cuda")
        B.dbw_preference_loss(self.shape, PAIRS, logits, tokens, start, self.logp(reference, context, tokens), None, BETA, 0.0, self.loss,
                              self.work, margin, dlogits=self.dlogits, status_out=self.status)
        self.round(context, hidden, lr)
        return self.loss.clone(), margin.mean()

    def policy(self, reference, lr, steps=2):
        """Tokens sampled from every worker's own model, rewarded by the teacher's log-probability; a few steps on one sample."""
        context = self.contexts()
        sampler = self.models(self.x[0].clone())
        tokens = self.sample(sampler.forward(context)[0])
        old, ref = self.logp(sampler, context, tokens), self.logp(reference, context, tokens)
        reward = self.logp(self.teacher, context, tokens).reshape(self.n, ROWS)
        advantage = ((reward - reward.mean(1, keepdim=True)) / (reward.std(1, keepdim=True) + 1e-6)).reshape(-1)
        kl = torch.empty(self.n, device="cuda")
        for _ in range(steps):
            logits, hidden = self.models(self.x[0]).forward(context)
            B.dbw_policy_loss(self.shape, logits, tokens, old, ref, advantage, None, CLIP_LOW, CLIP_HIGH, KL_COEF, self.loss, self.work,
                              kl_out=kl, dlogits=self.dlogits, status_out=self.status)
            self.round(context, hidden, lr)
        return reward.mean(), kl.mean()


def run(workers: int = 6, rounds: int = 40, seed: int = 1, experts: int = 0):
    """Curves of the three stages, as lists of floats, the status the losses left, and how many tokens a diverged model was to sample ("diverged": with any,
    the curves are no result)."""
    study = Study(workers, seed, experts)
    try:
        # Experts' weights multiply the step: with the first rates the ratio of a token with a negative advantage, which nothing bounds, overflows in the
        # second policy round.
        of_distill, of_rest = (2.0, 0.25) if experts else (8.0, 2.0)
        distill = [study.distill(of_distill) for _ in range(rounds)]
        reference = study.models(study.x[0].clone())
        preference = [study.preference(reference, of_rest) for _ in range(rounds)]
        reference = study.models(study.x[0].clone())
        policy = [study.policy(reference, of_rest) for _ in range(rounds)]
        torch.cuda.synchronize()
        B.dbw_check(study.h)
        return {"distill_loss": [v.mean().item() for v in distill],
                "preference_loss": [v[0].mean().item() for v in preference], "margin": [v[1].item() for v in preference],
                "reward": [v[0].item() for v in policy], "kl": [v[1].item() for v in policy],
                "status": int(study.status.item()), "diverged": int(study.diverged.item()), "params": study.x[0][:, :study.d].cpu().numpy()}
    finally:
        study.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workers", type=int, default=6)
    ap.add_argument("--rounds", type=int, default=40)
    ap.add_argument("--seed", type=int, default=1)
    ap.add_argument("--experts", type=int, default=0)
    args = ap.parse_args()
    out = run(args.workers, args.rounds, args.seed, args.experts)
    out.pop("params")
    print(json.dumps({k: [round(x, 5) for x in v] if isinstance(v, list) else v for k, v in out.items()}))
    if out["diverged"]:
        raise SystemExit(f"models diverged: {out['diverged']} tokens were sampled from no distribution")


if __name__ == "__main__":
    main()
