"""Asynchronous SGD of a small text classifier, learners and server on one GPU.

    python -m paper_1611_06213_amd.train_text [--learners 4] [--steps 200]

The model: `words` token ids look up their embeddings, which are dropped out and laid side by
side; a fully connected layer with ReLU and dropout; a fully connected layer to the
classes; softmax cross-entropy. With 9 words of 100 columns its first two layers are the embedding
and fc1 (900 -> 1000) of the Text-CNN workload.

Each learner, in its turn: pulls a replica, computes a gradient and pushes it. Weights are read
where they lie in the replica and gradients are written where they lie in the learner's row of
the server's memory: nothing is packed or copied. The fully connected layers run in 8-bit floating
point, their weights quantised once per pull; embeddings, biases and what the server holds do
not. Dropout stores no mask: the backward pass names the forward's seed and offset.

The data are synthetic: a class has words of its own, a text has some of them among random ones.
"""
from __future__ import annotations

import argparse
from typing import NamedTuple

import torch

from . import learner, ps


class Shape(NamedTuple):
    vocab: int = 5000
    words: int = 9
    dim: int = 100
    hidden: int = 1000
    classes: int = 50
    drop: float = 0.2

    def tensors(self):
        """(name, shape) in the flat vector's order."""
        return (("embedding", (self.vocab, self.dim)),
                ("fc1.weight", (self.hidden, self.words * self.dim)), ("fc1.bias", (self.hidden,)),
                ("fc2.weight", (self.classes, self.hidden)), ("fc2.bias", (self.classes,)))

    def params(self) -> int:
        return sum(torch.Size(s).numel() for _, s in self.tensors())

    def views(self, flat):
        """The model's tensors as views of a flat vector."""
        out, at = {}, 0
        for name, shape in self.tensors():
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out


class TextLearner:
    """One learner: a replica to pull into and a row for its gradient, both of the server's."""

    def __init__(self, shape: Shape, replica, row, seed: int):
        self.shape, self.replica, self.row, self.seed = shape, replica, row, seed
        self.w, self.g = shape.views(replica), shape.views(row)
        self.calls = 0

    def refresh(self) -> None:
        """After a pull: the layers' weights in 8 bits, as they are and (for the gradients of
        their inputs) transposed."""
        self.fc1, self.fc1_t = learner.quantize_fp8_both(self.w["fc1.weight"], square=True)
        self.fc2, self.fc2_t = learner.quantize_fp8_both(self.w["fc2.weight"], square=True)

    def drops(self):
        """The two dropouts of this call; others at the next."""
        d = [learner.Dropout(self.shape.drop, self.seed, 2 * self.calls + i) for i in range(2)]
        self.calls += 1
        return d

    def forward(self, tokens, drops=(None, None)):
        """(embedded words, hidden units, hidden units after dropout, logits)."""
        b = tokens.shape[0]
        x = learner.embedding(tokens.view(-1), self.w["embedding"], drop=drops[0], dtype=torch.bfloat16)
        x = x.view(b, -1)
        h = learner.linear_fp8(x, self.fc1, bias=self.w["fc1.bias"], relu=True)
        d = h if drops[1] is None else learner.dropout(h, drops[1])
        return x, h, d, learner.linear_fp8(d, self.fc2, bias=self.w["fc2.bias"], dtype=torch.float32)

    def gradient(self, tokens, labels):
        """Writes the gradient of the mean loss to the learner's row; returns the loss."""
        drops = self.drops()
        x, h, d, logits = self.forward(tokens, drops)
        b = tokens.shape[0]
        logp = torch.log_softmax(logits, 1)
        loss = -logp[torch.arange(b, device=logp.device), labels].mean()
        dz = logp.exp()
        dz[torch.arange(b, device=dz.device), labels] -= 1
        dz /= b
        g = self.g
        g["fc2.bias"].copy_(dz.sum(0))
        dd, _ = learner.linear_fp8_grad(d, dz, self.fc2_t, weight_out=g["fc2.weight"])
        dh = learner.dropout(dd, drops[1]) * (h > 0)
        g["fc1.bias"].copy_(dh.float().sum(0))
        dx, _ = learner.linear_fp8_grad(x, dh, self.fc1_t, weight_out=g["fc1.weight"])
        learner.embedding_grad(tokens.view(-1), dx.view(-1, self.shape.dim), self.shape.vocab,
                               drop=drops[0], out=g["embedding"])
        return loss


def initial_weights(shape: Shape, seed: int):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    w = torch.zeros(shape.params(), device="cuda")
    for name, v in shape.views(w).items():
        if name == "embedding":
            v.normal_(0.0, 1.0, generator=gen)
        elif v.dim() == 2:
            v.normal_(0.0, (2.0 / v.shape[1]) ** 0.5, generator=gen)
    return w


class Texts:
    """Synthetic texts: each class has eight words of its own, a third of a text's words."""

    def __init__(self, shape: Shape, seed: int):
        self.shape = shape
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.own = torch.randint(0, shape.vocab, (shape.classes, 8), generator=self.gen, device="cuda")

    def batch(self, n: int):
        s, gen = self.shape, self.gen
        labels = torch.randint(0, s.classes, (n,), generator=gen, device="cuda")
        tokens = torch.randint(0, s.vocab, (n, s.words), generator=gen, device="cuda")
        pick = self.own[labels[:, None], torch.randint(0, 8, (n, s.words), generator=gen, device="cuda")]
        here = torch.rand(n, s.words, generator=gen, device="cuda") < 1 / 3
        return torch.where(here, pick, tokens), labels


def train(shape: Shape, learners: int = 4, steps: int = 200, batch: int = 64, lr: float = 0.05,
          momentum: float = 0.0, seed: int = 1, verbose: bool = False):
    """Losses of `steps` pushes, the learners in turn: pull, gradient, push, apply."""
    srv = ps.ParameterServer(shape.params(), lr, momentum, queue_depth=1,
                             stream=torch.cuda.current_stream())
    try:
        srv.set_weights(initial_weights(shape, seed))
        rows = srv.alloc_rows(2 * learners)
        team = [TextLearner(shape, rows[2 * i], rows[2 * i + 1], seed + i) for i in range(learners)]
        texts = Texts(shape, seed)
        srv.pull_many(range(learners), [t.replica for t in team])
        for t in team:
            t.refresh()
        losses = []
        for step in range(steps):
            t = team[step % learners]
            losses.append(t.gradient(*texts.batch(batch)))
            srv.push(step % learners, t.row)
            srv.apply_pull([step % learners], [t.replica])
            t.refresh()
            if verbose and (step + 1) % 20 == 0:
                print(f"step {step + 1}: loss {float(torch.stack(losses[-20:]).mean()):.4f}", flush=True)
        srv.sync()
        return torch.stack(losses).cpu()
    finally:
        srv.close()


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--learners", type=int, default=4)
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--batch", type=int, default=64)
    p.add_argument("--lr", type=float, default=0.05)
    a = p.parse_args()
    losses = train(Shape(), a.learners, a.steps, a.batch, a.lr, verbose=True)
    print(f"loss of the first 20 pushes {float(losses[:20].mean()):.4f}, of the last 20 "
          f"{float(losses[-20:].mean()):.4f}", flush=True)


if __name__ == "__main__":
    main()
