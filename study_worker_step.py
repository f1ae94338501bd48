#!/usr/bin/env python3
"""Workers that train a small policy on what the receiver gives back: the whole way of a gradient, from tokens to tokens.

W workers hold the same parameters (a token table that is the output head too, a position table, one square matrix).  In an iteration each
samples answers to its own prompts, scores them under the policy as it is and under the one training began with, and takes a few
steps on them: embedding with dropout, a residual branch with dropout, logits, clipped policy loss with a KL term, and the way
back to one fp32 gradient vector.  The vectors are cut into packets, packets are lost, buckets that miss the tolerance are asked for
again, and every worker applies the mean that the receiver formed.

The right answer to a token is its successor, the reward one for it and zero otherwise, so the mean reward says whether all of it works:
it begins at one over the vocabulary and ends near one.

Sampling is torch's, and so are, unless --layers is given, the matrix products and the update; everything else is a kernel of the library.  With --layers the products are
the library's too, and the square matrix is updated by its mean gradient made orthogonal.  Prints one JSON object.  GPU required.
"""
from __future__ import annotations

import argparse
import json

import torch

import paper_2605_01989_amd as dblp

CLIP, KL = (0.2, 0.28), 0.002
MOST_PASSES = 1000              # of sending again in one round: more than a loss of 0.99 takes to a tolerance of 2 %
PROMPT = 4                      # leading tokens of a sequence that are given: no answer, no loss


class Policy:
    """The parameters as one fp32 vector, which is how the receiver returns a gradient, and views of its three tensors."""

    def __init__(self, vocab, seq, dim, seed):
        self.shapes = [(vocab, dim), (seq, dim), (dim, dim)]
        self.sizes = [a * b for a, b in self.shapes]
        self.n = sum(self.sizes)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.flat = torch.randn(self.n, generator=g, device="cuda").mul_(dim ** -0.5)
        self.table, self.positions, self.mix = self.views(self.flat)

    def views(self, flat):
        return [part.view(shape) for part, shape in zip(flat.split(self.sizes), self.shapes)]

    def buckets(self):
        """Offsets and counts of one bucket a tensor."""
        off = [0]
        for s in self.sizes[:-1]:
            off.append(off[-1] + s)
        return off, self.sizes


class Worker:
    """One worker's buffers, and its step.  Activations and logits are of type `dtype`; layers: the library's products and not torch's."""

    def __init__(self, policy, batch, seq, rank, p_drop, dtype=torch.bfloat16, layers=False):
        vocab, dim = policy.shapes[0]
        t, f = batch * seq, dict(device="cuda")
        self.layers = layers
        self.policy, self.rank, self.p_drop, self.batch, self.seq, self.dtype = policy, rank, p_drop, batch, seq, dtype
        self.gen = torch.Generator(device="cuda").manual_seed(1000 + rank)
        self.pos = torch.arange(seq, **f).repeat(batch)
        self.h, self.y, self.dz = (torch.empty(t, dim, dtype=dtype, **f) for _ in range(3))
        self.stats, self.old, self.ref = torch.empty(5, **f), torch.empty(t, **f), torch.empty(t, **f)
        self.grad = torch.empty(policy.n, **f)
        self.ws = torch.empty(max(dblp.embed_grad_workspace(t, vocab, dim), dblp.embed_grad_workspace(t, seq, dim), dblp.logits_workspace(t, vocab),
                                  dblp.linear_workspace(t, dim, vocab), dblp.linear_workspace(t, dim, dim)), dtype=torch.uint8, **f)

    def product(self, x, weight):
        """x weight^T, the weight in the activations' type."""
        if not self.layers:
            return x @ weight.T
        out = torch.empty(x.shape[0], weight.shape[0], dtype=x.dtype, device=x.device)
        dblp.linear(x, weight, out, self.ws)
        return out

    def product_grad(self, dy, x, weight, grad, base=None):
        """The gradient of x, on top of `base`; that of the weight in `grad`."""
        if not self.layers:
            grad.copy_(dy.T @ x)
            return dy @ weight if base is None else torch.addmm(base, dy, weight)
        dx = torch.empty_like(x)
        dblp.linear_grad_weight(dy, x, grad, self.ws)
        dblp.linear_grad_input(dy, weight, dx, self.ws, base=base)
        return dx

    def masks(self, step):
        """Of the sum of embeddings and of the residual branch; the seed is the worker's, a step draws two."""
        if step is None:
            return None, dblp.Drop(self.rank, 0, 0.0)
        return dblp.Drop(self.rank, 2 * step, self.p_drop), dblp.Drop(self.rank, 2 * step + 1, self.p_drop)

    def logits(self, params, step):
        """Of this worker's tokens, under the masks of a step (None: nothing is dropped, for sampling and scoring)."""
        table, positions, mix = params
        first, second = self.masks(step)
        dblp.embed(self.tokens, table, self.h, positions=self.pos, pos_table=positions, drop=first)
        dblp.dropout(self.product(self.h, mix.to(self.dtype)), self.y, second, residual=self.h)
        return self.product(self.y, table.to(self.dtype))

    def sample(self, start):
        """New prompts, answers to them, and both policies' scores."""
        p = self.policy
        vocab, t = p.shapes[0][0], self.batch * self.seq
        self.tokens = torch.randint(0, vocab, (t,), generator=self.gen, device="cuda")
        x = self.logits((p.table, p.positions, p.mix), None)
        # the largest of logits with Gumbel noise is a sample of their softmax
        answer = (x.float() - torch.empty(x.shape, device="cuda").exponential_(generator=self.gen).log()).argmax(1)
        self.targets = torch.where(self.pos < PROMPT, -1, answer)
        counted = self.targets >= 0
        dblp.token_logprobs(x, self.targets, self.old, self.ws)
        dblp.token_logprobs(self.logits(start, None), self.targets, self.ref, self.ws)
        reward = (answer == (self.tokens + 1) % vocab).float()
        mean = (reward * counted).sum() / counted.sum()
        self.advantages = (reward - mean) / (mean * (1 - mean) + 1e-3).sqrt()
        self.weights = counted.float() / counted.sum()
        return mean

    def gradient(self, step):
        """The loss' gradient with respect to the whole vector, in self.grad."""
        p = self.policy
        g_table, g_positions, g_mix = p.views(self.grad)
        first, second = self.masks(step)
        x = self.logits((p.table, p.positions, p.mix), step)
        dblp.policy_loss(x, self.targets, self.advantages, self.weights, self.stats, self.ws, old_logp=self.old, ref_logp=self.ref,
                         dlogits=x, clip=CLIP, kl_coef=KL)
        dy = self.product_grad(x, self.y, p.table.to(self.dtype), g_table)               # the table as the output head
        dblp.dropout(dy, self.dz, second)
        dh = self.product_grad(self.dz, self.h, p.mix.to(self.dtype), g_mix, base=dy)
        dblp.embed_grad(self.tokens, dh, g_table, self.ws, drop=first, base=g_table)     # and as the embedding, on top
        dblp.embed_grad(self.pos, dh, g_positions, self.ws, drop=first)
        return self.grad


class Receiver:
    """One communication round: packets, losses, what is asked for again, the mean."""

    def __init__(self, policy, workers, loss, bound_ppm, payload=366):
        if not 0 <= loss < 1:
            raise ValueError(f"loss: {loss} is no share of packets of which some arrive")
        off, cnt = policy.buckets()
        self.agg = dblp.Aggregator(workers, policy.n, payload, off, cnt)
        self.workers, self.loss, self.bound = workers, loss, bound_ppm
        n = workers * self.agg.n_pkts
        self.packets = torch.zeros(n * self.agg.stride, dtype=torch.uint8, device="cuda")
        self.src = torch.zeros(n, dtype=torch.int16, device="cuda")
        self.list = torch.empty(n, dtype=torch.int64, device="cuda")
        self.missing = torch.empty(workers * len(off), dtype=torch.int32, device="cuda")
        self.mean = torch.empty(policy.n, device="cuda")
        self.of_worker = torch.arange(workers, device="cuda").repeat_interleave(self.agg.n_pkts)
        self.gen = torch.Generator(device="cuda").manual_seed(77)

    def arrivals(self, of_worker):
        """A queue of the slots that are not lost, in any order: slot | worker << 32."""
        queue = torch.arange(of_worker.numel(), device="cuda") | of_worker << 32
        there = queue[torch.rand(queue.numel(), generator=self.gen, device="cuda") >= self.loss]
        return there[torch.randperm(there.numel(), generator=self.gen, device="cuda")]

    def round(self, number, grads):
        """(number of packets sent again, norm of the mean)"""
        agg, n = self.agg, self.workers * self.agg.n_pkts
        agg.begin_round(number)
        for w, g in enumerate(grads):
            agg.packetize(w, number, g, 0, 0, agg.n_pkts, self.packets, self.src, slot_base=w * agg.n_pkts)
        queue = self.arrivals(self.of_worker)
        agg.apply_arrivals_queue(self.packets, n, queue)
        again = 0
        for _ in range(MOST_PASSES):
            count, met, _ = agg.loss_account(self.bound, self.missing, self.list)
            if met:
                break
            again += count
            agg.packetize_list(number, grads, self.list, count, self.packets, self.src)
            queue = self.arrivals(self.list[:count] >> 32)
            if queue.numel():
                agg.apply_arrivals_queue(self.packets, count, queue)
        else:
            raise RuntimeError(f"round {number}: after {MOST_PASSES} passes of sending again {count} packets are missing still")
        agg.finalize(self.mean)
        return again, agg.phase_signal()[0]


class Update:
    """The step that a mean gradient is made into: its direction, clipped, or, of the square matrix and with `layers`, the nearly orthogonal matrix of a momentum of it."""

    def __init__(self, policy, rate, max_norm, layers, matrix_rate=0.02, momentum=0.8):
        self.policy, self.rate, self.max_norm, self.layers, self.matrix_rate, self.momentum = policy, rate, max_norm, layers, matrix_rate, momentum
        if layers:
            self.mean_mix = torch.zeros_like(policy.mix)
            self.ws = torch.empty(dblp.orthogonalize_workspace(1, *policy.mix.shape), dtype=torch.uint8, device="cuda")

    def __call__(self, mean, norm):
        p = self.policy
        step = -self.rate * min(1.0, self.max_norm / max(norm, 1e-30))
        if not self.layers:
            p.flat.add_(mean, alpha=step)
            return
        table, positions, mix = p.views(mean)
        p.table.add_(table, alpha=step)
        p.positions.add_(positions, alpha=step)
        self.mean_mix.mul_(self.momentum).add_(mix)
        dblp.orthogonalize(self.mean_mix, p.mix, self.ws, scale=-self.matrix_rate, base=p.mix)


def train(workers=4, iterations=40, steps=3, vocab=64, seq=32, dim=128, batch=64, p_drop=0.1, loss=0.1, bound_ppm=20_000, rate=4.0, max_norm=0.25, layers=False):
    policy = Policy(vocab, seq, dim, seed=1)
    start = [v.clone() for v in (policy.table, policy.positions, policy.mix)]
    group = [Worker(policy, batch, seq, rank, p_drop, layers=layers) for rank in range(workers)]
    update = Update(policy, rate, max_norm, layers)
    receiver = Receiver(policy, workers, loss, bound_ppm)
    out = dict(workers=workers, parameters=policy.n, packets_of_a_round=workers * receiver.agg.n_pkts, reward=[], kl=[], clipped=[], sent_again=0, rounds=0)
    for it in range(iterations):
        out["reward"].append(round(float(torch.stack([w.sample(start) for w in group]).mean()), 4))
        for k in range(steps):
            number = it * steps + k
            grads = [w.gradient(number) for w in group]
            again, norm = receiver.round(number + 1, grads)
            out["sent_again"] += again
            out["rounds"] += 1
            update(receiver.mean, norm)
        stats = torch.stack([w.stats for w in group]).mean(0).tolist()
        out["kl"].append(round(stats[2], 4))
        out["clipped"].append(round(stats[3] / max(stats[4], 1.0), 4))
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--iterations", type=int, default=40)
    ap.add_argument("--loss", type=float, default=0.1)
    ap.add_argument("--bound-ppm", type=int, default=20_000)
    ap.add_argument("--layers", action="store_true", help="the library's matrix products, and the square matrix' update made orthogonal")
    args = ap.parse_args()
    assert torch.cuda.is_available(), "needs a GPU"
    print(json.dumps(train(workers=args.workers, iterations=args.iterations, loss=args.loss, bound_ppm=args.bound_ppm, layers=args.layers)))


if __name__ == "__main__":
    main()
