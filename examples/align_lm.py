#!/usr/bin/env python3
"""A small language model taught what to prefer, by N data-parallel workers on one
GPU, every step from logits to updated parameters through libarctopk:

  logits -> the loss of preferred and rejected answers (--objective preference), or
            the clipped policy loss of answers that the model itself generated, with
            a KL term against where it began (--objective policy)
         -> each worker's gradient of all tensors (plain torch products)
         -> ARC-Top-K with EF21M -> norms and the clipping factor
         -> Muon for the hidden matrix, AdamW for all else

Prompts are a few tokens; an answer is liked the more of its tokens are even.

    python examples/align_lm.py [--objective policy] [--steps 60] [--workers 2]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2510_26709_amd as arc  # noqa: E402
from train_lm import Model  # noqa: E402


class Optimizer:
    """Muon for the tensors of two long sides but the embedding and the head, AdamW
    for the others; one norm and one clipping factor for all of them."""

    def __init__(self, model, device):
        vocab = max(r for r, _ in model.shapes)
        self.model = model
        self.matrices = [i for i, (r, c) in enumerate(model.shapes) if 1 < min(r, c)
                         and vocab not in (r, c)]
        self.rest = [i for i in range(len(model.shapes)) if i not in self.matrices]
        self.norms = arc.AdamW(model.sizes, device=device)
        self.muon = arc.Muon([model.shapes[i] for i in self.matrices], device=device)
        self.adamw = arc.AdamW([model.sizes[i] for i in self.rest], weight_decay=0.0,
                               device=device)

    def step(self, t, grad, lr, workers):
        total = self.norms.norm(grad, max_norm=1.0, scale=1.0 / workers).total
        x, g = self.model.views(self.model.x), self.model.views(grad)
        self.muon.step([x[i] for i in self.matrices], [g[i] for i in self.matrices], lr=lr,
                       factor=total)
        self.adamw.step(t, [x[i] for i in self.rest], [g[i] for i in self.rest], lr=lr,
                        factor=total)
        return total


def generate(model, prompts, length, gen):
    """Tokens sampled one after the other: [rows, prompt + length]."""
    tokens = prompts
    for _ in range(length):
        _, h = model.forward(tokens[:, -1])
        p = torch.softmax(model.logits(h), 1)
        tokens = torch.cat([tokens, torch.multinomial(p, 1, generator=gen)], 1)
    return tokens


def liking(tokens, prompt):
    return (tokens[:, prompt:] % 2 == 0).float().mean(1)


def rows_of(tokens, prompt):
    """Each token but the last as an input, the next one as what is given, -1 where
    that is the prompt's own."""
    given = tokens[:, 1:].clone()
    given[:, :prompt - 1] = -1
    return tokens[:, :-1].reshape(-1), given.reshape(-1)


def train(*, objective="policy", steps=60, workers=2, vocab=64, hidden=32, rows=32, prompt=3,
          length=9, keep=0.25, lr=0.02, device="cuda:0", log=lambda *a: None):
    """Returns how much the answers are liked before and after, and the totals of the
    last step."""
    device = torch.device(device)
    model = Model(vocab, hidden, device, seed=3)
    began = Model(vocab, hidden, device, seed=3)
    gen = torch.Generator(device=device).manual_seed(5)
    d, T = model.x.numel(), rows * (prompt + length - 1)
    tensors = [(r, c, r if r == 1 else math.ceil(keep * r)) for r, c in model.shapes]
    comp = arc.Compressor(d=d, N=workers, tensors=tensors, eta=0.5, seed=7, device=device)
    opt = Optimizer(model, device)
    head = arc.TokenLogProbs(V=vocab, rows=T, dtype="f32", device=device)
    grad = torch.empty(workers, d, device=device)
    h_state, g_state = torch.zeros(workers, d, device=device), torch.zeros(workers, d,
                                                                          device=device)
    offsets = torch.arange(rows + 1, device=device) * (prompt + length - 1)
    first = last = None
    for t in range(steps):
        liked = 0.0
        for i in range(workers):
            prompts = torch.randint(0, vocab, (rows, prompt), device=device, generator=gen)
            tokens = generate(model, prompts, length, gen)
            likes = liking(tokens, prompt)
            liked += float(likes.mean()) / workers
            if objective == "preference":  # the better half before the other one
                tokens = tokens[torch.argsort(likes, descending=True, stable=True)]
            x, given = rows_of(tokens, prompt)
            reference = head.score(began.logits(began.forward(x)[1]), given).logp
            e, h = model.forward(x)
            logits = model.logits(h)
            if objective == "preference":
                out = head.preference_loss(logits, given, offsets, ref_logp=reference, beta=0.3,
                                           scale=2.0 / rows, out=logits)
            else:
                old = head.score(logits, given).logp
                better = (likes - likes.mean()) / (likes.std() + 1e-6)
                out = head.policy_loss(
                    logits, given, better.repeat_interleave(prompt + length - 1), old_logp=old,
                    ref_logp=reference, kl_coef=0.02, entropy_coef=1e-3,
                    scale=1.0 / (rows * length), out=logits)
            model.backward(x, e, h, out.grad, grad[i])
        comp.step(t, grad, h_state, g_state)
        total = opt.step(t, g_state.sum(0), lr, workers)
        first, last = liked if first is None else first, liked
        if t % 10 == 0 or t == steps - 1:
            log(f"step {t}: liked {liked:.3f}, loss {float(out.totals[0]):.4f}, gradient norm "
                f"{float(total[0]):.3f}")
    comp.close()
    return first, last, out.totals


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--objective", choices=("policy", "preference"), default="policy")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=2)
    a = ap.parse_args()
    train(objective=a.objective, steps=a.steps, workers=a.workers,
          log=lambda *x: print(*x, flush=True))
