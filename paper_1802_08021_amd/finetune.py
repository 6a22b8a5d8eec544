"""Data-parallel fine-tuning with sparse gradients, all ranks on one GPU.

    python -m paper_1802_08021_amd.finetune

Every step takes the whole way of a gradient through the library: the loss of
each rank's tokens with its gradient (preference_loss, then policy_loss), the
largest entries of each bucket with error feedback (topk_bucketed, Alg. 1),
their sum over the ranks (ReduceCall), the norm of that sum and the AdamW step
over the model's tensors with 8-bit moments (AdamwCall).  The model between
them is a table of hidden vectors and an output matrix, whose products are
torch's: the next token is drawn from softmax(tanh(E[token]) @ W).

The task: the right answer to token x is (7 x + 3) mod V.  Pairs of answers
(right, wrong) come first, then answers drawn by the model itself with a
reward for each right one.
"""
from __future__ import annotations

import argparse

import torch

from . import sparcml as S


class Trainer:
    def __init__(self, vocab=256, hidden=64, ranks=4, tokens=256, state_bits=8, lr=2e-2, bucket=512, kb=16, seed=0,
                 device="cuda:0"):
        self.V, self.D, self.P, self.T = vocab, hidden, ranks, tokens
        self.dev = torch.device(device)
        self.gen = torch.Generator(device=self.dev).manual_seed(seed)
        self.sizes = [vocab * hidden, hidden * vocab, vocab]  # hidden vectors, output matrix, output bias
        n = sum(self.sizes)
        self.flat = torch.randn(n, device=self.dev, generator=self.gen) * 0.1
        self.flat[-vocab:] = 0
        self.E, self.W, self.b = self.views(self.flat)
        # one gradient, error and selection a rank; their sum is always dense
        # (delta 0+), so that the update's gradient tensors keep their place
        self.grads = torch.zeros(ranks, n, device=self.dev)
        self.select = S.TopkBucketedCall(torch.zeros_like(self.grads), self.grads, 1.0 / ranks, bucket, kb)
        self.reduce = S.ReduceCall([self.select.idx[r] for r in range(ranks)], n, 1e-12,
                                   vals=[self.select.val[r] for r in range(ranks)])
        params, grads = list(self.flat.split(self.sizes)), list(self.reduce.out_val.split(self.sizes))
        m, v, *scales = S.adamw_state(params, state_bits)
        kw = dict(zip(("m_scale", "v_scale"), scales))
        self.update = S.AdamwCall(params, grads, m, v, decay=[0.0, 0.01, 0.0], **kw)
        self.lr, self.steps = lr, 0
        self.start = self.flat.clone()  # the reference policy

    def views(self, flat):
        e, w, b = flat.split(self.sizes)
        return e.view(self.V, self.D), w.view(self.D, self.V), b

    def logits(self, x, flat=None):
        e, w, b = self.views(self.flat if flat is None else flat)
        h = torch.tanh(e[x])
        return h, h @ w + b

    def right(self, x):
        return (7 * x + 3) % self.V

    def draw(self, *shape):
        return torch.randint(0, self.V, shape, device=self.dev, generator=self.gen)

    def backward(self, rank, x, h, dlogits):
        """The loss' gradient from its logits' into the rank's row."""
        de, dw, db = self.views(self.grads[rank])
        de.zero_().index_add_(0, x, (dlogits @ self.W.t()) * (1 - h * h))
        torch.matmul(h.t(), dlogits, out=dw)
        torch.sum(dlogits, 0, out=db)

    def step(self):
        """Selection, sum over the ranks, norm, update."""
        self.select.run()
        self.reduce.run_async()
        clip = self.update.grad_norm(max_norm=1.0)
        self.steps += 1
        self.update.run(lr=self.lr, step=self.steps, beta2=0.99, clip=clip, seed=20180222)

    def preference_step(self):
        """Eight pairs a rank: the right answers against drawn ones.  Returns
        the mean of the ranks' stats (device)."""
        stats = []
        for rank in range(self.P):
            length = self.T // 16
            x = self.draw(8, length).repeat_interleave(2, 0)  # both answers to the same tokens
            y = self.right(x)
            y[1::2] = self.draw(8, length)
            x, y = x.reshape(-1), y.reshape(-1).int()
            h, z = self.logits(x)
            ref, _ = S.token_logprob(self.logits(x, self.start)[1], y)
            bounds = [i * length for i in range(17)]
            r = S.preference_loss(z, y, bounds, ref=ref, beta=0.1, dlogits="inplace")
            self.backward(rank, x, h, r["dlogits"])
            stats.append(r["stats"])
        self.step()
        return torch.stack(stats).mean(0)

    def policy_step(self):
        """Answers drawn by the model, rewarded where right.  Returns the mean
        of the ranks' stats and the mean reward (device)."""
        stats, rewards = [], []
        for rank in range(self.P):
            x = self.draw(self.T)
            h, z = self.logits(x)
            y = torch.multinomial(torch.softmax(z, 1), 1, generator=self.gen)[:, 0]
            reward = (y == self.right(x)).float()
            y = y.int()
            old, _ = S.token_logprob(z, y)
            ref, _ = S.token_logprob(self.logits(x, self.start)[1], y)
            weight = torch.full((self.T,), 1.0 / self.T, device=self.dev)
            r = S.policy_loss(z, y, old, reward - reward.mean(), weight, ref=ref, kl=1e-3, dlogits="inplace")
            self.backward(rank, x, h, r["dlogits"])
            stats.append(r["stats"])
            rewards.append(reward.mean())
        self.step()
        return torch.stack(stats).mean(0), torch.stack(rewards).mean()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--pairs-steps", type=int, default=60)
    ap.add_argument("--policy-steps", type=int, default=60)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args(argv)
    t = Trainer(ranks=a.ranks, state_bits=a.state_bits)
    for i in range(a.pairs_steps):
        stats = t.preference_step()
        if i % 10 == 9:
            loss, won, good, bad = stats.tolist()
            print(f"pairs  {i + 1:3d}: loss {loss:.4f}, in order {won:.2f}, rewards {good:+.3f} {bad:+.3f}, "
                  f"norm {float(t.update.out[0]):.3f}", flush=True)
    for i in range(a.policy_steps):
        stats, reward = t.policy_step()
        if i % 10 == 9:
            print(f"policy {i + 1:3d}: loss {float(stats[0]):+.4f}, KL {float(stats[2]):.4f}, "
                  f"right answers {float(reward):.3f}, norm {float(t.update.out[0]):.3f}", flush=True)


if __name__ == "__main__":
    main()
