"""A small transformer block trained by several learners whose gradients travel as AdaComp streams.

Each learner runs the block on its own batch (block.py: dropout, layer norm behind the residual add, attention softmax with
a relative position bias; the matrix products are torch's), packs the gradients of all parameters (norm weights and the bias
table among them) with adacomp_compress_multi, and adacomp_decompress_average_sgd_multi applies the sum of the streams to
the common weights.  The learners take turns on one GPU.  The task: sequences that repeat a random word; the block learns
to predict the next token from the one a word's length back.

    python -m paper_1712_02679_b200.block_step [--steps 300] [--learners 4]
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as B
from . import block

VOCAB, WORD = 24, 7


class Block:
    """Embedding, one block (attention and a feed-forward part, the norms behind the residual adds), an output product."""

    def __init__(self, width=128, heads=4, p=0.1, L_T=50, seed=0, device="cuda"):
        g = torch.Generator(device="cpu").manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, generator=g) / math.sqrt(shape[0])

        self.heads, self.p, self.L_T = heads, p, L_T
        self.plan = block.relpos(16, 32, bidirectional=False)
        values = {"embed": normal(VOCAB, width) * math.sqrt(VOCAB), "qkv": normal(width, 3 * width), "out": normal(width, width),
                  "up": normal(width, 4 * width), "down": normal(4 * width, width), "logits": normal(width, VOCAB),
                  "table": torch.zeros(16, heads)}
        for n in ("norm1", "norm2"):
            values[n + ".weight"], values[n + ".bias"] = torch.ones(width), torch.zeros(width)
        self.params = {k: v.to(device).requires_grad_() for k, v in values.items()}

    def loss(self, tokens: torch.Tensor, rng: block.Rng, site: int = 0, training: bool = True) -> torch.Tensor:
        """Mean loss of predicting the second half's tokens.  `site`: where this learner's dropouts start."""
        w = {k: v.to(torch.bfloat16) for k, v in self.params.items() if v.dim() == 2 and k != "table"}
        P, opt = self.params, dict(p=self.p, rng=rng, training=training)
        x = w["embed"][tokens[:, :-1]]
        b, n, d = x.shape
        q, k, v = (x @ w["qkv"]).view(b, n, 3, self.heads, d // self.heads).permute(2, 0, 3, 1, 4)
        probs = block.bias_softmax(q @ k.transpose(2, 3), P["table"], self.plan, scale=(d // self.heads) ** -0.5, causal=True,
                                   site=site, **opt)
        a = (probs @ v).transpose(1, 2).reshape(b, n, d) @ w["out"]
        y, _ = block.add_layer_norm(a, x, P["norm1.weight"], P["norm1.bias"], site=site + 1, **opt)
        f = block.dropout(torch.relu(y @ w["up"]), self.p, rng, site + 2, training) @ w["down"]
        y, _ = block.add_layer_norm(f, y, P["norm2.weight"], P["norm2.bias"], site=site + 3, **opt)
        half = n // 2
        logits = (y[:, half:] @ w["logits"]).float()
        return torch.nn.functional.cross_entropy(logits.reshape(-1, VOCAB), tokens[:, half + 1:].reshape(-1))


class Learners:
    """k learners' residues and streams, and the common weights' momentum."""

    def __init__(self, model: Block, k: int):
        self.model, self.k = model, k
        self.names = list(model.params)
        self.n = [model.params[m].numel() for m in self.names]
        dev = model.params[self.names[0]].device
        self.residue = [[torch.zeros(n, device=dev) for n in self.n] for _ in range(k)]
        self.packed = [[torch.empty(B.adacomp_packed_capacity(n, model.L_T), dtype=torch.uint8, device=dev) for n in self.n]
                       for _ in range(k)]
        self.count = [[torch.zeros(2, dtype=torch.int64, device=dev) for _ in self.n] for _ in range(k)]
        self.momentum = [torch.zeros(n, device=dev) for n in self.n]

    def step(self, batches, rng: block.Rng, lr: float, mu: float = 0.9) -> float:
        """One synchronous step: batches[l] is learner l's.  Returns the learners' mean loss."""
        total = torch.zeros((), device=rng.state.device)
        params = [self.model.params[m] for m in self.names]
        for l in range(self.k):
            loss = self.model.loss(batches[l], rng, site=8 * l)
            grads = torch.autograd.grad(loss, params)
            total += loss.detach() / self.k
            B.adacomp_compress_multi([dict(grad=g.reshape(-1).contiguous(), residue=self.residue[l][t], n=self.n[t],
                                           L_T=self.model.L_T, packed_out=self.packed[l][t], count_out=self.count[l][t])
                                      for t, g in enumerate(grads)], len(grads))
        with torch.no_grad():
            B.adacomp_decompress_average_sgd_multi([self.packed[l][t] for t in range(len(params)) for l in range(self.k)], self.k,
                                                   [q.detach().view(-1) for q in params], self.momentum, self.n,
                                                   [self.model.L_T] * len(params), len(params), lr, mu)
        rng.advance()
        return float(total)

    def sent(self) -> float:
        """Elements the last step sent, of all."""
        return sum(int(c[0]) for row in self.count for c in row) / (self.k * sum(self.n))


def batch(size: int, length: int, gen: torch.Generator, device="cuda") -> torch.Tensor:
    word = torch.randint(0, VOCAB, (size, WORD), generator=gen)
    return word.repeat(1, -(-(length + 1) // WORD))[:, :length + 1].to(device)


def train(steps=300, k=4, size=16, length=64, lr=0.02, seed=0, report=None):
    """Losses of every step."""
    model, rng = Block(seed=seed), block.Rng(seed + 1)
    learners = Learners(model, k)
    gen = torch.Generator().manual_seed(seed + 2)
    losses = []
    for s in range(steps):
        losses.append(learners.step([batch(size, length, gen) for _ in range(k)], rng, lr))
        if report and (s % 25 == 0 or s + 1 == steps):
            report(f"step {s:4d}  loss {losses[-1]:.4f}  sent {100 * learners.sent():.2f} %")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--learners", type=int, default=4)
    a = ap.parse_args()
    train(a.steps, a.learners, report=print)
