#!/usr/bin/env python3
"""A small language model trained by N data-parallel workers on one GPU, every
step from logits to updated parameters through libarctopk:

  logits -> log probabilities of the given tokens and their gradient
         -> each worker's gradient of all tensors (plain torch products)
         -> ARC-Top-K with EF21M (the compressed all-reduce's payload)
         -> norms and the clipping factor of the workers' sum -> AdamW

The data is a synthetic Markov chain, whose entropy is the loss that no model
gets under; the perplexity at the end is of tokens that no step saw.

    python examples/train_lm.py [--steps 300] [--workers 4] [--state f8]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2510_26709_amd as arc  # noqa: E402


class Chain:
    """Tokens of a Markov chain with a few likely successors of each."""

    def __init__(self, vocab, seed, device):
        gen = torch.Generator(device=device).manual_seed(seed)
        logits = torch.randn(vocab, vocab, device=device, generator=gen) * 3.0
        self.p = torch.softmax(logits, 1)
        self.gen = gen

    def sample(self, rows, length):
        x = torch.empty(rows, length + 1, dtype=torch.int64, device=self.p.device)
        x[:, 0] = torch.randint(0, self.p.shape[0], (rows,), device=self.p.device,
                                generator=self.gen)
        for k in range(length):
            x[:, k + 1] = torch.multinomial(self.p[x[:, k]], 1, generator=self.gen)[:, 0]
        return x[:, :-1].reshape(-1), x[:, 1:].reshape(-1)

    def entropy(self):
        return float(-(self.p * self.p.log()).sum(1).mean())


class Model:
    """Embedding, one hidden layer, head: tensors side by side in one flat
    vector, the layout that the compressor and AdamW share."""

    def __init__(self, vocab, hidden, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.shapes = [(vocab, hidden), (hidden, hidden), (1, hidden), (vocab, hidden)]
        self.sizes = [a * b for a, b in self.shapes]
        self.x = torch.randn(sum(self.sizes), device=device, generator=gen) / math.sqrt(hidden)

    def views(self, flat):
        return [t.view(s) for t, s in zip(torch.split(flat, self.sizes), self.shapes)]

    def forward(self, tokens):
        E, W, b, _ = self.views(self.x)
        e = E[tokens]
        h = torch.tanh(e @ W + b)
        return e, h

    def logits(self, h):
        return h @ self.views(self.x)[3].t()

    def backward(self, tokens, e, h, dlogits, grad):
        """The gradient of all tensors, into a flat vector."""
        _, W, _, U = self.views(self.x)
        gE, gW, gb, gU = self.views(grad)
        torch.mm(dlogits.t(), h, out=gU)
        dh = (dlogits @ U) * (1 - h * h)
        torch.mm(e.t(), dh, out=gW)
        gb.copy_(dh.sum(0, keepdim=True))
        # (sorted sums: their order, and with it a run's every bit, is the same each time)
        gE.zero_().index_put_((tokens,), dh @ W.t(), accumulate=True)


def train(*, steps=300, workers=4, vocab=501, hidden=128, rows=32, length=16, keep=0.2, lr=1e-2,
          max_norm=1.0, state="f32", device="cuda:0", log=lambda *a: None):
    """Returns (first loss, last loss, perplexity, the chain's entropy)."""
    device = torch.device(device)
    data = Chain(vocab, 1, device)
    model = Model(vocab, hidden, device)
    d, N, T = model.x.numel(), workers, rows * length
    tensors = [(r, c, r if r == 1 else math.ceil(keep * r)) for r, c in model.shapes]
    comp = arc.Compressor(d=d, N=N, tensors=tensors, eta=0.5, seed=7, device=device)
    opt = arc.AdamW(model.sizes, state=state, weight_decay=[0.01, 0.01, 0.0, 0.01], seed=7,
                    device=device)
    head = arc.TokenLogProbs(V=vocab, rows=T, dtype="f32", top=3, device=device)
    grad = torch.empty(N, d, device=device)
    h_state, g_state = torch.zeros(N, d, device=device), torch.zeros(N, d, device=device)
    per_token = torch.full((T,), -1.0 / T, device=device)  # of the mean loss, by log probability
    first = last = None
    for t in range(steps):
        total = torch.zeros((), device=device)
        for i in range(N):
            tokens, targets = data.sample(rows, length)
            e, h = model.forward(tokens)
            logits = model.logits(h)
            out = head.loss(logits, targets, per_token, out=logits)  # in place of the logits
            model.backward(tokens, e, h, out.grad, grad[i])
            total -= out.logp.mean() / N
        comp.step(t, grad, h_state, g_state)
        G = g_state.sum(0)  # what every worker holds after the exchange
        norms = opt.norm(G, max_norm=max_norm, scale=1.0 / N)
        opt.step(t, model.x, G, lr=lr * min(1.0, (t + 1) / 20), factor=norms.total)
        if t == 0 or t == steps - 1 or t % 50 == 0:
            last = float(total)
            first = last if first is None else first
            log(f"step {t}: loss {last:.4f}, gradient norm {float(norms.total[0]):.3f}")
    tokens, targets = data.sample(rows, length)
    scores = head.score(model.logits(model.forward(tokens)[1]), targets)
    perplexity = float(torch.exp(-scores.logp.mean()))
    hit = float((scores.top_ids == targets[:, None]).any(1).float().mean())
    log(f"held out: perplexity {perplexity:.2f} (the chain's own {math.exp(data.entropy()):.2f}), "
        f"entropy {float(scores.entropy.mean()):.3f}, given token among the three likeliest "
        f"{100 * hit:.0f}% of the time")
    comp.close()
    return first, last, perplexity, data.entropy()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--state", choices=("f32", "f8"), default="f32")
    a = ap.parse_args()
    train(steps=a.steps, workers=a.workers, state=a.state, log=lambda *x: print(*x, flush=True))
