"""A head on the batched chain LSTM, trained by preferences and by a clipped policy loss.

Sentences of different lengths run as one mini-batch of chain-LSTM graphs; on the states h of all words:

    z = layer_norm(h, w, b)
    u = gelu(z W + c) + z                       linear, with its residual
    x = u O                                     linear: the vocabulary logits
    lp = logprobs(x, the word after each)

Of every two neighbouring sentences the first is preferred (preference_loss against the log probabilities at the
start); then each sentence gets an advantage and the words are tuned by policy_loss.  The gradients go back through
logprobs_grad, linear_grad and layer_norm_grad to w, b, W, c and O; the cells stay as drawn.

    python examples/preferred_words.py --instances 16 --vocab 5000 --steps 20
"""
import argparse
import pathlib
import sys

sys.path.insert(0, str(pathlib.Path(__file__).resolve().parent.parent))

import numpy as np
import torch

from paper_2302_03851_amd import edb, head, tokens, workloads


class Head:
    """Layer norm, one hidden layer and the vocabulary's product."""

    def __init__(self, hidden, vocab, seed, device):
        g = torch.Generator(device=device).manual_seed(seed)
        self.w = torch.ones(hidden, device=device)
        self.b = torch.zeros(hidden, device=device)
        self.W = torch.randn((hidden, hidden), generator=g, device=device) / hidden ** 0.5
        self.c = torch.zeros(hidden, device=device)
        self.O = torch.randn((hidden, vocab), generator=g, device=device) / hidden ** 0.5

    def logits(self, h):
        """The logits, and what the way back needs."""
        z = head.layer_norm(h, self.w, self.b)
        u = head.linear(z.out, self.W, self.c, "gelu", z.out, keep=True)
        return head.linear(u.out, self.O).out, (h, z, u)

    def gradients(self, kept, dx):
        """Gradients of w, b, W, c and O from the logits'."""
        h, z, u = kept
        top = head.linear_grad(u.out, self.O, dx, dbias=False)
        mid = head.linear_grad(z.out, self.W, top.dx, "gelu", u.pre)
        low = head.layer_norm_grad(h, z.stats, mid.dx + top.dx, self.w, dx=False)
        return [low.dweight, low.dbias, mid.dweight, mid.dbias, top.dweight]

    def step(self, gradients, rate):
        for t, g in zip((self.w, self.b, self.W, self.c, self.O), gradients):
            t.add_(g, alpha=-rate)


def preferred(model, h, ids, first, reference, beta):
    """The pairs' losses and the gradients of their mean; without a reference, of the log probabilities themselves."""
    x, kept = model.logits(h)
    r = tokens.logprobs(x, ids)
    pairs = (first.numel() - 1) // 2
    weight = torch.full((pairs,), 1.0 / pairs, device=h.device)
    p = tokens.preference_loss(r.logprob, reference, first, beta=beta, mean=True, ids=ids, weight=weight)
    dx = tokens.logprobs_grad(x, ids, r.stats, g_logprob=p.g_logprob, out=x)
    return r.logprob, p, model.gradients(kept, dx)


def tuned(model, h, ids, first, old, reference, advantage, kl):
    """The sentences' losses and the gradients of their mean."""
    x, kept = model.logits(h)
    r = tokens.logprobs(x, ids)
    weight = torch.full((advantage.numel(),), 1.0 / advantage.numel(), device=h.device)
    p = tokens.policy_loss(r.logprob, old, first, advantage, (0.2, 0.28), reference, kl, ids=ids, weight=weight)
    dx = tokens.logprobs_grad(x, ids, r.stats, g_logprob=p.g_logprob, out=x)
    return r.logprob, p, model.gradients(kept, dx)


def states(instances, vocab, device):
    """The states of all words of `instances` sentences, the word after each (-1 after the last) and the sentences' first words."""
    w = workloads.make_config(1, instances=instances)
    f = edb.Forward(w, device=device)
    f.run()
    h = f.arena_h[torch.as_tensor(np.asarray(f.plan.slot).astype(np.int64), device=device)].float()
    g = torch.Generator(device=device).manual_seed(1)
    # the nodes of a sentence are neighbours
    begins = torch.as_tensor(np.asarray(w.child_idx[w.child_ptr[:-1]]) < 0, device=device)
    word = torch.randint(0, vocab, (w.n_nodes,), generator=g, device=device, dtype=torch.int32)
    last = torch.cat([begins[1:], begins.new_ones(1)])
    ids = torch.where(last, torch.full_like(word, -1), word.roll(-1))
    first = torch.cat([torch.nonzero(begins)[:, 0], torch.tensor([w.n_nodes], device=device)]).to(torch.int32)
    return h, ids, first


def run(instances=16, vocab=5000, steps=20, rate=0.2, device="cuda:0", report=print):
    """Prefers, then tunes; returns the mean loss at every step of both."""
    torch.cuda.set_device(torch.device(device))
    h, ids, first = states(instances, vocab, device)
    model = Head(h.shape[1], vocab, 2, device)
    reference = tokens.logprobs(model.logits(h)[0], ids).logprob
    preferences, tunings = [], []
    for _ in range(steps):
        _, p, gradients = preferred(model, h, ids, first, reference, 0.5)
        model.step(gradients, rate)
        preferences.append(p.loss.mean())
    advantage = torch.where(torch.arange(first.numel() - 1, device=device) % 2 == 0, 1.0, -1.0)
    old = tokens.logprobs(model.logits(h)[0], ids).logprob
    clipped = 0
    for _ in range(steps):
        _, p, gradients = tuned(model, h, ids, first, old, reference, advantage, 0.02)
        model.step(gradients, rate / 4)
        tunings.append(p.loss.mean())
        clipped = p.clipped.sum()
    preferences, tunings = torch.stack(preferences).tolist(), torch.stack(tunings).tolist()
    report(f"{instances} sentences, {h.shape[0]} words of {vocab}")
    report(f"preference loss {preferences[0]:.4f} -> {preferences[-1]:.4f}")
    report(f"policy loss {tunings[0]:.4f} -> {tunings[-1]:.4f}, {int(clipped)} words clipped, "
           f"divergence {float(p.kl.mean()):.4f} a word")
    return preferences, tunings


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--instances", type=int, default=16)
    p.add_argument("--vocab", type=int, default=5000)
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args()
    run(a.instances, a.vocab, a.steps)
