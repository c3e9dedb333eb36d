"""Asynchronous SGD of a small text classifier, learners and server on one GPU.

    python -m paper_1611_06213_amd.train_text [--learners 4] [--steps 200] [--blocks 2] [--adamw 8]

The model: `words` token ids look up their embeddings, which are dropped out and laid side by
side; a fully connected layer with ReLU and dropout; `blocks` residual blocks, each a fully
connected layer with ReLU between a norm before it and one after it, gated (their weights: fc2 1000 ->
1000 of the Text-CNN workload); a fully connected layer to the classes; softmax cross-entropy. With 9
words of 100 columns its first two layers are the embedding and fc1 (900 -> 1000) of that workload.

Each learner, in its turn: pulls a replica, computes a gradient and pushes it. Weights are read
where they lie in the replica and gradients are written where they lie in the learner's row of
the server's memory: nothing is packed or copied. The fully connected layers run in 8-bit floating
point, their weights quantised once per pull; embeddings, biases and what the server holds do
not. Dropout stores no mask: the backward pass names the forward's seed and offset.

With --adamw each learner makes an AdamW step of its gradient, with states of its own in 8 or 32
bits, and pushes that: the server subtracts it. At the end a replica answers: `Answers` has its
fully connected layers in 8-bit integers.

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
    blocks: int = 0

    def tensors(self):
        """(name, shape) in the flat vector's order."""
        out = (("embedding", (self.vocab, self.dim)),
               ("fc1.weight", (self.hidden, self.words * self.dim)), ("fc1.bias", (self.hidden,)),
               ("fc2.weight", (self.classes, self.hidden)), ("fc2.bias", (self.classes,)))
        for i in range(self.blocks):
            out += ((f"block{i}.weight", (self.hidden, self.hidden)),
                    *((f"block{i}.{name}", (self.hidden,)) for name in ("bias", "before", "after", "gate")))
        return out

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
        self.adamw = None

    def use_adamw(self, bits: int, decay: float = 0.01) -> None:
        """From now on `step` makes AdamW steps of the row's gradients, weights (but not biases and
        vectors) decaying."""
        self.adamw = learner.AdamW([self.w[k] for k in self.w], [self.g[k] for k in self.w],
                                   decay=[decay if v.dim() == 2 else 0.0 for v in self.w.values()],
                                   bits=bits, push=True, seed=self.seed)

    def refresh(self) -> None:
        """After a pull: the layers' weights in 8 bits, as they are and (for the gradients of
        their inputs) transposed."""
        self.fc1, self.fc1_t = learner.quantize_fp8_both(self.w["fc1.weight"], square=True)
        self.fc2, self.fc2_t = learner.quantize_fp8_both(self.w["fc2.weight"], square=True)
        self.blocks = [learner.quantize_fp8_both(self.w[f"block{i}.weight"], square=True)
                       for i in range(self.shape.blocks)]

    def drops(self):
        """The two dropouts of this call; others at the next."""
        d = [learner.Dropout(self.shape.drop, self.seed, 2 * self.calls + i) for i in range(2)]
        self.calls += 1
        return d

    def vectors(self, i: int, of=None):
        """A block's gate, its norm after it and the norm before the next one (None: there is none), of the weights
        or of the views `of`."""
        of = self.w if of is None else of
        return {"gate": of[f"block{i}.gate"], "after": of[f"block{i}.after"], "before": of.get(f"block{i + 1}.before")}

    def stack(self, s, layer):
        """The residual blocks: what they leave of the stream s, and for each (its stream, its input, its output),
        with `layer(i, z)` as its layer."""
        kept = []
        z = learner.rms_norm(s, self.w["block0.before"]) if self.shape.blocks else None
        for i in range(self.shape.blocks):
            y = layer(i, z)
            kept.append((s, z, y))
            s, z = learner.residual_norm(s, y, **self.vectors(i))
        return s, kept

    def forward(self, tokens, drops=(None, None), kept=None):
        """(embedded words, hidden units, hidden units after dropout, logits); `kept` gets what `stack` keeps, and the
        stream behind the blocks."""
        b = tokens.shape[0]
        x = learner.embedding(tokens.view(-1), self.w["embedding"], drop=drops[0], dtype=torch.bfloat16)
        x = x.view(b, -1)
        h = learner.linear_fp8(x, self.fc1, bias=self.w["fc1.bias"], relu=True)
        d = h if drops[1] is None else learner.dropout(h, drops[1])
        s, of_blocks = self.stack(d, lambda i, z: learner.linear_fp8(
            z, self.blocks[i][0], bias=self.w[f"block{i}.bias"], relu=True))
        if kept is not None:
            kept += [*of_blocks, s]
        return x, h, d, learner.linear_fp8(s, self.fc2, bias=self.w["fc2.bias"], dtype=torch.float32)

    def stack_gradient(self, kept, ds):
        """Writes the blocks' gradients to the row, from that of the stream behind them; returns that of the stream
        before them."""
        dz, g, after = None, self.g, kept[-1]
        for i in reversed(range(self.shape.blocks)):
            s, z, y = kept[i]
            outs = {f"{k}_out": v for k, v in self.vectors(i, g).items()}
            ds, dy, *_ = learner.residual_norm_grad(after, y, ds, dz, **self.vectors(i), **outs)
            dy = dy * (y > 0)
            g[f"block{i}.bias"].copy_(dy.float().sum(0))
            dz, _ = learner.linear_fp8_grad(z, dy, self.blocks[i][1], weight_out=g[f"block{i}.weight"])
            after = s
        if dz is not None:
            ds, _ = learner.rms_norm_grad(after, self.w["block0.before"], dz, stream_grad=ds,
                                          weight_out=g["block0.before"])
        return ds

    def gradient(self, tokens, labels):
        """Writes the gradient of the mean loss to the learner's row; returns the loss."""
        drops = self.drops()
        kept = []
        x, h, d, logits = self.forward(tokens, drops, kept)
        b = tokens.shape[0]
        logp = torch.log_softmax(logits, 1)
        loss = -logp[torch.arange(b, device=logp.device), labels].mean()
        dz = logp.exp()
        dz[torch.arange(b, device=dz.device), labels] -= 1
        dz /= b
        g = self.g
        g["fc2.bias"].copy_(dz.sum(0))
        ds, _ = learner.linear_fp8_grad(kept[-1], dz, self.fc2_t, weight_out=g["fc2.weight"])
        dd = self.stack_gradient(kept, ds)
        dh = learner.dropout(dd, drops[1]) * (h > 0)
        g["fc1.bias"].copy_(dh.float().sum(0))
        dx, _ = learner.linear_fp8_grad(x, dh, self.fc1_t, weight_out=g["fc1.weight"])
        learner.embedding_grad(tokens.view(-1), dx.view(-1, self.shape.dim), self.shape.vocab,
                               drop=drops[0], out=g["embedding"])
        return loss

    def step(self, lr: float) -> None:
        """With AdamW: the row's gradient becomes the step that the server is to make."""
        if self.adamw is not None:
            self.adamw.step(lr)


class Answers(TextLearner):
    """A replica that answers: no gradients, its fully connected layers in 8-bit integers, so that an answer does not
    depend on the others of its batch."""

    def __init__(self, shape: Shape, replica):
        super().__init__(shape, replica, replica, 0)

    def refresh(self) -> None:
        self.fc1 = learner.quantize_int8(self.w["fc1.weight"])
        self.fc2 = learner.quantize_int8(self.w["fc2.weight"])
        self.blocks = [learner.quantize_int8(self.w[f"block{i}.weight"]) for i in range(self.shape.blocks)]

    def logits(self, tokens):
        b = tokens.shape[0]
        x = learner.embedding(tokens.view(-1), self.w["embedding"], dtype=torch.bfloat16).view(b, -1)
        d = learner.linear_int8(x, self.fc1, bias=self.w["fc1.bias"], relu=True)
        s, _ = self.stack(d, lambda i, z: learner.linear_int8(
            z, self.blocks[i], bias=self.w[f"block{i}.bias"], relu=True))
        return learner.linear_int8(s, self.fc2, bias=self.w["fc2.bias"], dtype=torch.float32)


def initial_weights(shape: Shape, seed: int):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    w = torch.zeros(shape.params(), device="cuda")
    for name, v in shape.views(w).items():
        if name == "embedding":
            v.normal_(0.0, 1.0, generator=gen)
        elif v.dim() == 2:
            v.normal_(0.0, (2.0 / v.shape[1]) ** 0.5, generator=gen)
        elif name.endswith((".before", ".after")):
            v.fill_(1.0)
        elif name.endswith(".gate"):
            v.fill_(0.1)
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
          momentum: float = 0.0, seed: int = 1, verbose: bool = False, adamw: int = 0, answers: int = 0):
    """Losses of `steps` pushes, the learners in turn: pull, gradient, push, apply; with `answers` also the share of
    so many new texts whose class a replica in 8-bit integers then names. `adamw`: the bits of the learners' states,
    0 for the server's own steps."""
    # a pushed step is subtracted as it is
    srv = ps.ParameterServer(shape.params(), 1.0 if adamw else lr, 0.0 if adamw else momentum, queue_depth=1,
                             stream=torch.cuda.current_stream())
    try:
        srv.set_weights(initial_weights(shape, seed))
        rows = srv.alloc_rows(2 * learners)
        team = [TextLearner(shape, rows[2 * i], rows[2 * i + 1], seed + i) for i in range(learners)]
        texts = Texts(shape, seed)
        srv.pull_many(range(learners), [t.replica for t in team])
        for t in team:
            t.refresh()
            if adamw:
                t.use_adamw(adamw)
        losses = []
        for step in range(steps):
            t = team[step % learners]
            losses.append(t.gradient(*texts.batch(batch)))
            t.step(lr)
            srv.push(step % learners, t.row)
            srv.apply_pull([step % learners], [t.replica])
            t.refresh()
            if verbose and (step + 1) % 20 == 0:
                print(f"step {step + 1}: loss {float(torch.stack(losses[-20:]).mean()):.4f}", flush=True)
        right = None
        if answers:
            # any learner's replica will do: the first one's, of the weights as they are now
            srv.pull_many([0], [team[0].replica])
            replica = Answers(shape, team[0].replica)
            replica.refresh()
            tokens, labels = texts.batch(answers)
            right = (replica.logits(tokens).argmax(1) == labels).float().mean()
        srv.sync()
        losses = torch.stack(losses).cpu()
        return (losses, float(right)) if answers else losses
    finally:
        srv.close()


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--learners", type=int, default=4)
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--batch", type=int, default=64)
    p.add_argument("--blocks", type=int, default=0, help="residual blocks")
    p.add_argument("--adamw", type=int, choices=(8, 32), default=0, help="AdamW learners, bits of their states")
    p.add_argument("--lr", type=float, help="0.05, with --adamw 0.001")
    p.add_argument("--answers", type=int, default=0, help="texts to classify at the end, in 8-bit integers")
    a = p.parse_args()
    lr = a.lr if a.lr is not None else 0.001 if a.adamw else 0.05
    got = train(Shape(blocks=a.blocks), a.learners, a.steps, a.batch, lr, verbose=True, adamw=a.adamw,
                answers=a.answers)
    losses = got[0] if a.answers else got
    if a.answers:
        print(f"{a.answers} texts answered in 8-bit integers: {100 * got[1]:.1f}% right", flush=True)
    print(f"loss of the first 20 pushes {float(losses[:20].mean()):.4f}, of the last 20 "
          f"{float(losses[-20:].mean()):.4f}", flush=True)


if __name__ == "__main__":
    main()
