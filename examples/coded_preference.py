#!/usr/bin/env python3
"""Trains a small language-model head by pipelined gradient coding with the operators of
paper_2607_20739_amd.ops: dropout, token log-probabilities, the preference loss, the policy loss.

  python examples/coded_preference.py                       PGC-FR, 4 workers, one straggler a step
  python examples/coded_preference.py --scheme CR --n 6 --c 3 --steps 60

n workers hold c partitions of preference pairs each (Sec. III).  At step t >= 1 a worker evaluates the
one in slot (t - 1) mod c, keeps the latest gradient of each, and sends their coded sum; the master
ignores the stragglers, decodes and updates (Sec. IV-A, V-B).  A second phase goes on with the
policy loss on the preferred answers, scored by the first phase's model.

A partition's gradient must be the same whichever worker evaluates it.  Hence dropout draws its mask
from the step and the token's number in the data set, and every loss is a fixed-order sum over its own
rows.  With FR the decoded gradient then is the same for every set of stragglers, to the last bit.

The model is features -> hidden (ReLU, dropout, residual) -> vocabulary, in bf16 products by torch.
The data is synthetic: a fixed random teacher writes the preferred answers, chance the others.
"""

import argparse
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2607_20739_amd as P  # noqa: E402
from paper_2607_20739_amd import ops  # noqa: E402


class Pairs:
    """A partition's pairs: tokens' features, targets (-1 in prompts), sequence bounds, numbers."""

    def __init__(self, k, pairs, longest, width, vocab, teacher, device):
        g = torch.Generator(device=device)
        g.manual_seed(1000 + k)
        lengths = torch.randint(3, longest + 1, (2 * pairs,), generator=g, device=device)
        ends = lengths.cumsum(0)
        self.offsets = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
        rows = int(ends[-1])
        self.x = torch.randn(rows, width, generator=g, device=device).to(torch.bfloat16)
        right = (self.x.float() @ teacher).argmax(1)
        other = torch.randint(0, vocab, (rows,), generator=g, device=device)
        at = torch.arange(rows, device=device)
        seq = torch.searchsorted(ends, at, right=True)
        self.preferred = seq % 2 == 0
        prompt = at == self.offsets.long()[seq]          # one prompt token per sequence
        self.targets = torch.where(prompt, -1, torch.where(self.preferred, right, other)).to(torch.int32)
        self.numbers = at + k * (1 << 20)                # of the tokens in the whole data set
        self.pairs = pairs


class Head:
    """Parameters as one fp32 vector, as the coded gradients are."""

    def __init__(self, width, vocab, device):
        g = torch.Generator(device=device)
        g.manual_seed(7)
        self.width, self.vocab = width, vocab
        w1 = torch.randn(width, width, generator=g, device=device) / width ** 0.5
        w2 = torch.randn(width, vocab, generator=g, device=device) * (0.1 / width ** 0.5)
        self.w = torch.cat([w1.reshape(-1), w2.reshape(-1)])

    def logits(self, w, x, drop=None):
        """drop: (p, seed, the tokens' numbers), or None to evaluate without dropout."""
        n = self.width * self.width
        w1, w2 = w[:n].view(self.width, -1).to(torch.bfloat16), w[n:].view(self.width, -1).to(torch.bfloat16)
        h = torch.relu(x @ w1)
        h = h + x if drop is None else ops.dropout(h, drop[0], drop[1], residual=x, row_ids=drop[2])
        return h @ w2

    def gradient(self, data, loss, drop):
        """The partition's gradient: loss(logits) gives the logits'."""
        w = self.w.detach().clone().requires_grad_()
        z = self.logits(w, data.x, drop)
        value, dz = loss(z.detach())
        z.backward(dz)
        return value, w.grad


class Coded:
    """The workers' rings and the master's decode on the library's placement and coefficients.

    With each_worker every worker evaluates its own copy of a partition and keeps a ring of its own.  Otherwise one
    evaluation serves all holders of a partition, which gives the same words as long as its gradient does not depend on
    who computes it.
    """

    def __init__(self, scheme, n, c, q, device, each_worker=False):
        self.n, self.c, self.scheme, self.each_worker = n, c, scheme, each_worker
        self.ctx = P.pgc_init(scheme, n, c, 4)           # for its tables alone
        P.pgc_configure(self.ctx, "lsq", n, 4)
        self.placement = P.pgc_placement(self.ctx, n, c)
        # [slot][worker], or, for all holders together, [slot][partition].
        self.ring = torch.zeros(c, n, q, device=device)
        self.t = 0

    def place(self, worker, slot):
        """Where the worker's copy in that slot lies in the ring."""
        return worker if self.each_worker else int(self.placement[worker][slot])

    def word(self, worker):
        return sum(self.ring[slot, self.place(worker, slot)] for slot in range(self.c))

    def step(self, evaluate, straggler_mask):
        """One step: evaluate(worker, partition) -> gradient; returns the decoded gradient."""
        slots = range(self.c) if self.t == 0 else [(self.t - 1) % self.c]
        fresh = {}
        for slot in slots:
            for worker in range(self.n):
                k = int(self.placement[worker][slot])
                if self.each_worker:
                    self.ring[slot, worker] = evaluate(worker, k)
                    continue
                if k not in fresh:
                    fresh[k] = evaluate(worker, k)
                # FR: a group's members share their copies; CR: the slot is one worker's own.
                for s in range(self.c) if self.scheme == "FR" else [slot]:
                    self.ring[s, k] = fresh[k]
        survivors, d, scale = P.pgc_decode_coeffs(self.ctx, straggler_mask, self.n)
        ghat = torch.zeros_like(self.ring[0, 0])
        for j, weight in zip(survivors, d):
            if weight != 0:
                ghat += float(weight) * self.word(j)
        self.t += 1
        return ghat * scale

    def close(self):
        P.pgc_destroy(self.ctx)


def train(scheme="FR", n=4, c=2, steps=40, policy_steps=20, pairs=6, longest=12, width=64, vocab=1000, lr=0.2, policy_lr=0.1, p=0.1,
          mask_seed=3, device="cuda", each_worker=False):
    """Both phases; returns {"preference": losses, "accuracy": of the pairs, "policy": losses, "w": parameters,
    "words": each worker's word of each step, where each evaluates its own}."""
    g = torch.Generator(device=device)
    g.manual_seed(1)
    teacher = torch.randn(width, vocab, generator=g, device=device)
    data = [Pairs(k, pairs, longest, width, vocab, teacher, device) for k in range(n)]
    head = Head(width, vocab, device)
    # The reference model's scores are fixed: the model before the first step.
    reference = [ops.token_logprobs(head.logits(head.w, part.x), part.targets)[0] for part in data]
    out = {"preference": [], "policy": [], "words": []}

    def run(count, first, loss_of, rate, name):
        coded = Coded(scheme, n, c, head.w.numel(), device, each_worker)
        try:
            for t in range(count):
                mask = P.pgc_make_mask(mask_seed, first + t, P.PGC_POLICY_EXACT, n, c - 1)
                values = []

                def evaluate(worker, k):
                    drop = (p, P.pgc_splitmix64(99, first + t), data[k].numbers)
                    value, grad = head.gradient(data[k], loss_of(k), drop)
                    values.append(value)
                    return grad
                head.w -= rate * coded.step(evaluate, mask)
                out[name].append(float(torch.stack(values).mean()))
                if each_worker:
                    out["words"].append([coded.word(j) for j in range(n)])
        finally:
            coded.close()

    def preference_of(k):
        part = data[k]

        def loss(z):
            value, _, _, dz = ops.preference_loss(z, part.targets, part.offsets, reference[k], beta=0.5, scale=1.0 / pairs)
            return value.mean(), dz
        return loss

    run(steps, 0, preference_of, lr, "preference")
    margins = [ops.preference_loss(head.logits(head.w, part.x), part.targets, part.offsets, reference[k], gradient=False)[1]
               for k, part in enumerate(data)]
    out["accuracy"] = float((torch.cat(margins) > 0).float().mean())

    old = [ops.token_logprobs(head.logits(head.w, part.x), part.targets)[0] for part in data]

    def policy_of(k):
        part = data[k]
        advantages = torch.where(part.preferred, 1.0, -0.2)

        def loss(z):
            value, _, dz = ops.policy_loss(z, part.targets, old[k], advantages, ref_logprobs=reference[k], clip_high=0.28,
                                           kl=0.01, scale=1.0 / len(part.x))
            return value.mean(), dz
        return loss

    run(policy_steps, steps, policy_of, policy_lr, "policy")
    out["w"] = head.w
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--scheme", choices=["FR", "CR"], default="FR")
    ap.add_argument("--n", type=int, default=4)
    ap.add_argument("--c", type=int, default=2)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--policy-steps", type=int, default=20)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--each-worker", action="store_true", help="every worker evaluates its own copy of a partition")
    args = ap.parse_args()
    out = train(args.scheme, args.n, args.c, args.steps, args.policy_steps, vocab=args.vocab, each_worker=args.each_worker)
    print(json.dumps({"scheme": args.scheme, "n": args.n, "c": args.c, "preference_first": out["preference"][0],
                      "preference_last": out["preference"][-1], "pairs_ranked_right": out["accuracy"],
                      "policy_first": out["policy"][0], "policy_last": out["policy"][-1]}))


if __name__ == "__main__":
    main()
