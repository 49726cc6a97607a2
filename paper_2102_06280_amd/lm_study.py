"""Small language models of N workers trained through the library's losses on logits and its rounds.

Three stages, one after the other, on synthetic tokens: distillation from a fixed teacher's top logits, a preference
loss on pairs of answers, and a clipped policy loss with a KL term on sampled tokens.  Every round is the same: the
workers' logits, a loss of dbw_losses.h with the logits' gradient, from that the models' gradients, the selection of
neighbours from the round's response times, and dbw_round with the gradients as ext_grads.  Losses, gradients of the
logits, selection, averaging and local step are the library's; the model (a hidden layer on the last two tokens) and
its backward pass are the caller's, a few products of torch in fp32.

    python -m paper_2102_06280_amd.lm_study [--workers 6] [--rounds 40]
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
        dhidden = torch.bmm(dlogits, self.out.contiguous()) * (1 - hidden * hidden)
        for k, into in enumerate((g.first, g.second)):
            which = torch.nn.functional.one_hot(context[..., k], VOCAB).float()
            into.copy_(torch.bmm(which.transpose(1, 2).contiguous(), dhidden))


class Study:
    def __init__(self, workers: int, seed: int = 1):
        self.n = workers
        self.ld = inputs.pad_ld(D)
        g = np.random.default_rng(seed)
        self.times = g
        rowptr, colidx = inputs.graph_ring(workers) if workers > 2 else inputs.graph_complete(workers)
        self.backups = torch.from_numpy((np.diff(rowptr) > 1).astype(np.int32)).cuda()       # one backup worker where there are two
        self.h = B.dbw_create(rowptr, colidx, workers, D, ld=self.ld)
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        draw = lambda rows, spread: torch.randn(rows, self.ld, device="cuda", generator=self.gen) * spread
        self.teacher_rows = draw(1, 1.5).expand(workers, -1).contiguous()
        self.teacher = Models(self.teacher_rows)
        self.x = [draw(workers, 0.3), torch.zeros(workers, self.ld, device="cuda")]
        self.grads = torch.zeros(workers, self.ld, device="cuda")
        # what the losses need: a shape, scratch memory, outputs
        self.shape = B.make_logits(workers, ROWS, VOCAB, B.TYPE_F32, scale=SCALE)
        self.work = torch.empty(B.dbw_loss_work_bytes(self.shape), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dlogits = torch.empty(workers, ROWS, VOCAB, device="cuda")
        self.loss = torch.empty(workers, device="cuda")

    def close(self):
        B.dbw_destroy(self.h)

    def contexts(self):
        return torch.randint(0, VOCAB, (self.n, ROWS, 2), device="cuda", generator=self.gen)

    def sample(self, logits):
        p = torch.softmax(logits * SCALE, -1).reshape(-1, VOCAB)
        return torch.multinomial(p, 1, generator=self.gen)[:, 0].int()

    def logp(self, models, context, tokens):
        out = torch.empty(self.n * ROWS, device="cuda")
        B.dbw_token_logp(self.shape, models.forward(context)[0], tokens, out, self.work, status_out=self.status)
        return out

    def round(self, context, hidden, lr):
        """From the logits' gradient to the parameters after the round."""
        Models(self.x[0]).backward(context, hidden, self.dlogits, self.grads)
        t = torch.from_numpy(self.times.standard_exponential(self.n).astype(np.float32)).cuda()
        B.dbw_select(self.h, t, self.backups)
        B.dbw_round(self.h, self.x[0], self.x[1], lr, ext_grads=self.grads)
        self.x.reverse()

    def distill(self, lr):
        context = self.contexts()
        logits, hidden = Models(self.x[0]).forward(context)
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
        logits, hidden = Models(self.x[0]).forward(context)
        margin = torch.empty(self.n * PAIRS, device="cuda")
        B.dbw_preference_loss(self.shape, PAIRS, logits, tokens, start, self.logp(reference, context, tokens), None, BETA, 0.0, self.loss,
                              self.work, margin, dlogits=self.dlogits, status_out=self.status)
        self.round(context, hidden, lr)
        return self.loss.clone(), margin.mean()

    def policy(self, reference, lr, steps=2):
        """Tokens sampled from every worker's own model, rewarded by the teacher's log-probability; a few steps on one sample."""
        context = self.contexts()
        sampler = Models(self.x[0].clone())
        tokens = self.sample(sampler.forward(context)[0])
        old, ref = self.logp(sampler, context, tokens), self.logp(reference, context, tokens)
        reward = self.logp(self.teacher, context, tokens).reshape(self.n, ROWS)
        advantage = ((reward - reward.mean(1, keepdim=True)) / (reward.std(1, keepdim=True) + 1e-6)).reshape(-1)
        kl = torch.empty(self.n, device="cuda")
        for _ in range(steps):
            logits, hidden = Models(self.x[0]).forward(context)
            B.dbw_policy_loss(self.shape, logits, tokens, old, ref, advantage, None, CLIP_LOW, CLIP_HIGH, KL_COEF, self.loss, self.work,
                              kl_out=kl, dlogits=self.dlogits, status_out=self.status)
            self.round(context, hidden, lr)
        return reward.mean(), kl.mean()


def run(workers: int = 6, rounds: int = 40, seed: int = 1):
    """Curves of the three stages, as lists of floats, and the status the losses left."""
    study = Study(workers, seed)
    try:
        distill = [study.distill(8.0) for _ in range(rounds)]
        reference = Models(study.x[0].clone())
        preference = [study.preference(reference, 2.0) for _ in range(rounds)]
        reference = Models(study.x[0].clone())
        policy = [study.policy(reference, 2.0) for _ in range(rounds)]
        torch.cuda.synchronize()
        B.dbw_check(study.h)
        return {"distill_loss": [v.mean().item() for v in distill],
                "preference_loss": [v[0].mean().item() for v in preference], "margin": [v[1].item() for v in preference],
                "reward": [v[0].item() for v in policy], "kl": [v[1].item() for v in policy],
                "status": int(study.status.item()), "params": study.x[0][:, :D].cpu().numpy()}
    finally:
        study.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workers", type=int, default=6)
    ap.add_argument("--rounds", type=int, default=40)
    ap.add_argument("--seed", type=int, default=1)
    args = ap.parse_args()
    out = run(args.workers, args.rounds, args.seed)
    out.pop("params")
    print(json.dumps({k: [round(x, 5) for x in v] if isinstance(v, list) else v for k, v in out.items()}))


if __name__ == "__main__":
    main()
