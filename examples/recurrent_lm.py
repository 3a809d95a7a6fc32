"""A recurrent language model on the word table, trained and asked.

The model reads a sentence from its first word on and scores every word of the
vocabulary as the next one:

  e_t = dropout(E[w_t])                      rows gathered with dropout
  h_t = a_t h_{t-1} + (1 - a_t) x_t          a_t = sigmoid(Wg e_t + bg), x_t = Wx e_t
  s_t(w) = h_t . O[w]

and is trained as the window ranker is: the word that comes next has to outscore a
word drawn at random by a margin of one, max(0, 1 - s_t(next) + s_t(random)),
averaged over the words.  One step of SGD is Context.dropout, Context.recurrence,
Context.recurrence_backward, Context.dropout_backward and Context.scatter_add on
both tables; the small dense products are torch's.

Answering keeps one state per live sequence: Context.recurrence_step, the scores of
all words, and Context.logits, which takes words that were said before down, allows
what a grammar allows, and picks.

The corpus is planted: sentences of a few to forty words in which a word is followed
by the one that a fixed permutation gives for it, nine times out of ten, and the
permutation leads from words of even number to words of odd number and back.

  python examples/recurrent_lm.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_1404_1521_amd as pg


class Corpus:
    """Sentences of the planted language."""

    def __init__(self, V: int, seed: int):
        self.V, self.rng = V, np.random.default_rng(seed)
        even, odd = np.arange(0, V, 2), np.arange(1, V, 2)
        self.next = np.empty(V, np.int64)
        self.next[even] = self.rng.permutation(odd)
        self.next[odd] = self.rng.permutation(even)

    def batch(self, sentences: int):
        """Words, the word that follows each, and the sentences' offsets (int32)."""
        words, follows, offsets = [], [], [0]
        for n in self.rng.integers(2, 41, sentences):
            w = int(self.rng.integers(0, self.V))
            for _ in range(n):
                words.append(w)
                w = int(self.next[w]) if self.rng.random() < 0.9 else \
                    int(self.rng.integers(0, self.V))
                follows.append(w)
            offsets.append(len(words))
        return [torch.tensor(a, dtype=torch.int32, device="cuda")
                for a in (words, follows, offsets)]


class Model:
    def __init__(self, V: int, d: int, max_tokens: int, max_live: int, seed: int = 0):
        self.V, self.d = V, d
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(*shape, device="cuda").normal_(0, std, generator=gen)

        self.E, self.O = normal(V, d, std=0.3), normal(V, d, std=0.3)
        self.Wg, self.Wx = normal(d, d, std=d ** -0.5), normal(d, d, std=d ** -0.5)
        self.bg = torch.zeros(d, device="cuda")
        # the model shape of the context is the window ranker's and matters to nothing here
        self.ctx = pg.Context(V, 16, 1, 8, max_batch=1, max_scatter=2 * max_tokens, max_rows=V)
        self.ctx.reserve_recurrence(max_tokens, d)
        self.ctx.reserve_logits(max_live, V)
        self.seed = seed

    def train_step(self, words, follows, offsets, random, lr: float, p: float, step: int):
        """One step of SGD in place; returns the mean hinge loss (a device scalar)."""
        ctx, n = self.ctx, words.shape[0]
        e = ctx.dropout(self.E, p, self.seed, site=step, ids=words)
        gate, x = torch.addmm(self.bg, e, self.Wg.t()), e @ self.Wx.t()
        h, _ = ctx.recurrence(gate, x, offsets)

        good, bad = self.O[follows.long()], self.O[random.long()]
        margin = 1 - (h * (good - bad)).sum(1)
        # the hinge's derivative, over the mean; 0 where the margin is met
        hit = (margin > 0).float().unsqueeze(1) / n
        dh = hit * (bad - good)
        dgood = -hit * h

        dgate, dx, _ = ctx.recurrence_backward(gate, x, h, dh, offsets)
        de = dgate @ self.Wg + dx @ self.Wx
        dE = ctx.dropout_backward(de, p, self.seed, site=step)
        dWg, dWx, dbg = dgate.t() @ e, dx.t() @ e, dgate.sum(0)

        ctx.scatter_add(self.E, words, dE, -lr)
        ctx.scatter_add(self.O, torch.cat([follows, random]), torch.cat([dgood, -dgood]), -lr)
        self.Wg -= lr * dWg
        self.Wx -= lr * dWx
        self.bg -= lr * dbg
        return margin.clamp(min=0).mean()

    def scores(self, words, state):
        """The states after one more word of every live sequence, updated in place, and
        the scores of all words as the next one."""
        e = self.E[words.long()]
        h, _ = self.ctx.recurrence_step(torch.addmm(self.bg, e, self.Wg.t()), e @ self.Wx.t(), state,
                                        last=state)
        return h @ self.O.t()

    def generate(self, words, length: int, repetition: float = 1.0, presence: float = 0.0,
                 mask=None, mask_of=None):
        """Continues every sequence of one word by `length` words: the best allowed one,
        words that were said before taken down.  mask: rows of allowed words, as
        Context.logits has them; mask_of(words) says which row each sequence is in.
        Returns [sequences][1 + length] words and the log-probabilities of the choices."""
        n = words.shape[0]
        state = torch.zeros(n, self.d, device="cuda")
        history = torch.full((n, 1 + length), -1, dtype=torch.int32, device="cuda")
        history[:, 0] = words
        logp = torch.empty(n, length, device="cuda")
        penalties = dict(repetition=torch.full((n,), repetition, device="cuda"),
                         presence=torch.full((n,), presence, device="cuda"))
        for k in range(length):
            said = torch.full((n,), k + 1, dtype=torch.int32, device="cuda")
            out, words, lse = self.ctx.logits(
                self.scores(words, state), history=history, lengths=said, mask=mask,
                mask_rows=None if mask is None else mask_of(words), **penalties)
            history[:, k + 1] = words
            logp[:, k] = out.gather(1, words.long().unsqueeze(1))[:, 0] - lse
        return history, logp


def bits(allowed):
    """Rows of truth values as rows of mask words."""
    n, V = allowed.shape
    full = np.zeros((n, (V + 31) // 32 * 32), bool)
    full[:, :V] = allowed
    return torch.from_numpy(np.packbits(full, axis=1, bitorder="little").view(np.int32)).cuda()


def main(steps: int = 400, V: int = 200, d: int = 64, sentences: int = 64, quiet: bool = False):
    """Trains, then generates.  Returns the first and the last hundred steps' mean losses,
    the share of the next words that the model names, and what it generated."""
    corpus = Corpus(V, seed=1)
    model = Model(V, d, max_tokens=40 * sentences, max_live=64)
    gen = torch.Generator(device="cuda").manual_seed(2)
    losses = []
    for step in range(steps):
        words, follows, offsets = corpus.batch(sentences)
        random = torch.randint(0, V, words.shape, device="cuda", generator=gen).to(torch.int32)
        losses.append(model.train_step(words, follows, offsets, random, lr=20.0, p=0.1, step=step))
        if not quiet and step % 50 == 49:
            print(f"step {step + 1}: loss {float(torch.stack(losses[-50:]).mean()):.4f}", flush=True)
    losses = torch.stack(losses).tolist()

    start = torch.arange(0, 64, dtype=torch.int32, device="cuda") % V
    said, _ = model.generate(start, 8)
    named = float((said[:, 1:].cpu().numpy() == corpus.next[said[:, :-1].cpu().numpy()]).mean())
    # the grammar's two states: odd words after even ones, even words after odd ones; and
    # nothing said twice
    allowed = np.stack([np.arange(V) % 2 == 1, np.arange(V) % 2 == 0])
    held, logp = model.generate(start, 20, presence=1e4, mask=bits(allowed),
                                mask_of=lambda w: (w % 2).to(torch.int32))
    status = model.ctx.status()
    if status != pg.OK:
        raise RuntimeError(f"device error word: {status}")
    if not quiet:
        print(f"loss {np.mean(losses[:50]):.4f} -> {np.mean(losses[-50:]):.4f}; "
              f"{100 * named:.1f}% of the next words named")
        print("held to the grammar, nothing twice:", held[0].tolist())
    return losses, named, held.cpu().numpy(), logp.cpu().numpy()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=400)
    main(ap.parse_args().steps)
