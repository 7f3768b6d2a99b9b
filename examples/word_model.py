"""A word model on the batched chain LSTM, from ids to scores, with every token operator.

Sentences of different lengths run as one mini-batch of chain-LSTM graphs.  The
model predicts each next word:

    x      = embed(ids, E)                      written straight into the graphs' input rows
    h      = the chain LSTM's states            (edb.Forward; its weights and E stay as drawn)
    z      = h + embed(ids, B)                  B: a trained row per word
    logits = z O                                O: the trained output weights

A teacher of the same form scores the words first; the 16 best of each place are
kept (logprobs), and the student learns them:

    distill                                     loss and gradient of the logits in one call
    dz = dlogits O^T,  dO = z^T dlogits         products of torch
    embed_grad(ids, dz)                         gradient of B

Then it is tuned on the words that came (logprobs, logprobs_grad, with a small
reward for entropy) and asked for the words that may follow each sentence.

    python examples/word_model.py --instances 16 --vocab 5000 --steps 30
"""
import argparse
import pathlib
import sys

sys.path.insert(0, str(pathlib.Path(__file__).resolve().parent.parent))

import numpy as np
import torch

from paper_2302_03851_amd import edb, tokens, workloads


class WordModel:
    def __init__(self, w, vocab, seed, device):
        g = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.encoder = vocab, edb.Forward(w, device=device)
        self.slot = torch.as_tensor(np.asarray(self.encoder.plan.slot).astype(np.int64), device=device)
        dt, H = self.encoder.tdt, w.hidden
        # scales that the gates and the logits can carry: x of order 1, logits of order 3
        self.inputs = torch.randn((vocab, w.in_dim), generator=g, device=device).to(dt)
        self.skip = torch.randn((vocab, H), generator=g, device=device) * 0.5
        self.out = torch.randn((H, vocab), generator=g, device=device) * (6.0 / H ** 0.5)

    def features(self, ids):
        """z [nodes, hidden]: the state after each word, and the word's own row."""
        tokens.embed(ids, self.inputs, out=self.encoder.x)
        self.encoder.run()
        return self.encoder.arena_h[self.slot].float() + tokens.embed(ids, self.skip)

    def logits(self, z):
        return torch.mm(z, self.out)

    def step(self, ids, z, dlogits, rate):
        """One step down the gradients of B and O."""
        dz = torch.mm(dlogits, self.out.t().contiguous())
        self.out.add_(torch.mm(z.t().contiguous(), dlogits), alpha=-rate)
        tokens.embed_grad(ids, dz, self.vocab, scale=-rate, out=self.skip, accumulate=True)


def run(instances=16, vocab=5000, steps=30, kept=16, temperature=2.0, rate=0.3, device="cuda:0", report=print):
    """Distils, tunes and asks; returns the mean loss at every step of both."""
    torch.cuda.set_device(torch.device(device))
    w = workloads.make_config(1, instances=instances)
    n = w.n_nodes
    g = torch.Generator(device=device).manual_seed(1)
    ids = torch.randint(0, vocab, (w.x.shape[0],), generator=g, device=device, dtype=torch.int32)
    # the word after each, none after a sentence's last; the nodes of a sentence are neighbours
    first = torch.as_tensor(np.asarray(w.child_idx[w.child_ptr[:-1]]) < 0, device=device)
    last = torch.cat([first[1:], first.new_ones(1)])
    row = torch.as_tensor(np.asarray(w.x_row).astype(np.int64), device=device)
    word = ids[row]
    following = torch.where(last, torch.full_like(word, -1), word.roll(-1))

    teacher, student = WordModel(w, vocab, 2, device), WordModel(w, vocab, 3, device)
    student.inputs = teacher.inputs
    best = tokens.logprobs(teacher.logits(teacher.features(ids)), None, 1.0, kept)

    distilled, tuned = [], []
    weight = torch.full((n,), 1.0 / n, device=device)      # of the mean; the rate grows with the number of words
    for _ in range(steps):
        z = student.features(ids)
        x = student.logits(z)
        t = tokens.distill(x, best.top_ids, best.top_logprobs, temperature, weight)
        student.step(word, z, t.dlogits, rate * n / 4)
        distilled.append(t.loss.mean())
    places = (following >= 0).sum()
    up = (1.0 / places).expand(n).contiguous()
    for _ in range(steps):
        z = student.features(ids)
        x = student.logits(z)
        r = tokens.logprobs(x, following)
        dx = tokens.logprobs_grad(x, following, r.stats, r.entropy, -up, -0.01 * up, out=x)
        student.step(word, z, dx, rate * n / 4)
        tuned.append(-r.logprob.sum() / places)

    # the words that may follow each sentence, and how open the question is
    x = student.logits(student.features(ids)[last])
    answers = tokens.logprobs(x, None, 1.0, 5)
    distilled, tuned = torch.stack(distilled).tolist(), torch.stack(tuned).tolist()
    report(f"{instances} sentences, {n} words of {vocab}")
    report(f"distillation loss {distilled[0]:.4f} -> {distilled[-1]:.4f}")
    report(f"loss of the words that came {tuned[0]:.4f} -> {tuned[-1]:.4f}")
    for i in range(min(3, x.shape[0])):
        said = ", ".join(f"{v} ({p:.3f})" for v, p in zip(answers.top_ids[i].tolist(), answers.top_logprobs[i].exp().tolist()))
        report(f"after sentence {i}: {said}; entropy {answers.entropy[i].item():.3f}")
    return distilled, tuned


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--instances", type=int, default=16)
    p.add_argument("--vocab", type=int, default=5000)
    p.add_argument("--steps", type=int, default=30)
    a = p.parse_args()
    run(a.instances, a.vocab, a.steps)
