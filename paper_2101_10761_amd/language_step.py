"""A training run of a small language model whose workers use its operators together: `python -m paper_2101_10761_amd.language_step`.

Words become rows of a table (sidco_embedding), elements are dropped (sidco_dropout), one hidden layer goes into the residual, and
the table, which is the decoder's weight too, gives the losses of the next words and the gradients (sidco_cross_entropy,
sidco_cross_entropy_grad).  On the way back the lookup's gradient is added to the decoder's in the one buffer that the exchange of
dense_step takes (sidco_embedding_grad with accumulate): dense in 4 bits with error feedback, or sparse as selected pairs.  The
hidden layer multiplies in 4 bits (dense_step.Layer) or in fp32, its weights move by the orthogonalised momentum.

The workers are simulated one after the other on one GPU, each with its own text and residual.  The text is synthetic: a word is
followed by one of a few others of its own most of the time, and some places are padding.
"""
from __future__ import annotations

import argparse

from . import binding as sidco
from .dense_step import Exchange4Bit, ExchangeSparse, Layer


class Fp32Layer:
    """The same as dense_step.Layer with torch's products."""

    def __init__(self, weight, batch: int):
        pass

    def forward(self, x, weight):
        self.x, self.weight = x, weight
        return x @ weight.t()

    def backward(self, dy, weight_grad):
        weight_grad.copy_(dy.t() @ self.x)
        return dy @ self.weight


class Model:
    """Losses of n words' successors, and the gradients, written into views of one flat buffer."""

    def __init__(self, vocab: int, dim: int, n: int, p: float, seed: int, device, hidden: str = "4bit"):
        import torch
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device=device)  # noqa: E731
        self.table, self.weight = normal(vocab, dim) / dim ** 0.5, normal(dim, dim) / dim ** 0.5
        self.scale, self.p, self.seed, self.n, self.blocks = dim ** 0.5, p, seed, n, 0
        self.layer = (Layer if hidden == "4bit" else Fp32Layer)(self.weight, n)
        rows = lambda: torch.empty(n, dim, device=device)  # noqa: E731
        self.x, self.h, self.y = rows(), rows(), rows()
        self.dy, self.dh, self.dx = rows(), rows(), rows()
        self.loss, self.lse, self.loss_grad = (torch.empty(n, device=device) for _ in range(3))

    def forward(self, words, targets):
        """The losses of `targets`; every call drops other elements."""
        n, dim = self.x.shape
        self.words, self.targets = words, targets
        self.first, self.second = self.blocks, self.blocks + sidco.sidco_dropout_blocks(n, dim)
        self.blocks = self.second + sidco.sidco_dropout_blocks(n, dim)
        sidco.sidco_embedding(self.table, words, self.x, scale=self.scale)
        sidco.sidco_dropout(self.x, self.x, self.p, self.seed, offset=self.first)
        self.h.copy_(self.layer.forward(self.x, self.weight)).relu_()
        sidco.sidco_dropout(self.h, self.y, self.p, self.seed, offset=self.second, residual=self.x)
        sidco.sidco_cross_entropy(self.y, self.table, targets, self.loss, self.lse)
        return self.loss

    def backward(self, table_grad, weight_grad):
        """The gradients of the mean over the targets that are no padding."""
        valid = (self.targets >= 0) & (self.targets < len(self.table))
        self.loss_grad.copy_(1.0 / valid.sum().clamp(min=1))
        sidco.sidco_cross_entropy_grad(self.y, self.table, self.targets, self.lse, self.loss_grad, self.dy, table_grad, loss=self.loss)
        sidco.sidco_dropout(self.dy, self.dh, self.p, self.seed, offset=self.second)
        self.dh.mul_(self.h > 0)
        self.dx.copy_(self.layer.backward(self.dh, weight_grad)).add_(self.dy)
        sidco.sidco_dropout(self.dx, self.dx, self.p, self.seed, offset=self.first)
        sidco.sidco_embedding_grad(self.dx, self.words, table_grad, scale=self.scale, accumulate=True)


def text(n: int, vocab: int, generator, padding: float = 0.05):
    """Words and the words that follow them."""
    import torch
    dev = generator.device
    words = torch.randint(0, vocab, (n,), generator=generator, device=dev)
    after = (words * 31 + torch.randint(0, 3, (n,), generator=generator, device=dev)) % vocab
    chance = torch.rand(n, generator=generator, device=dev)
    after = torch.where(chance < 0.1, torch.randint(0, vocab, (n,), generator=generator, device=dev), after)
    hidden = torch.rand(n, generator=generator, device=dev) < padding
    return torch.where(hidden, -1, words), torch.where(hidden, -1, after)


def train(exchange: str = "4bit", workers: int = 2, steps: int = 60, n: int = 700, vocab: int = 1000, dim: int = 192, p: float = 0.1,
          lr: float = 1.0, delta: float = 0.1, seed: int = 0, hidden: str = "4bit") -> dict:
    """Trains and returns {"losses": [...], "bytes": of a worker's message, "gradient_bytes": of the gradient in float32}."""
    import torch
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    model = Model(vocab, dim, n, p, seed, dev, hidden)
    d = vocab * dim + dim * dim
    grad, mean, momentum = torch.zeros(d, device=dev), torch.zeros(d, device=dev), torch.zeros(dim, dim, device=dev)
    views = lambda flat: (flat[: vocab * dim].view(vocab, dim), flat[vocab * dim:].view(dim, dim))  # noqa: E731
    swap = Exchange4Bit(workers, d, dev) if exchange == "4bit" else ExchangeSparse(workers, d, dev, delta)
    losses = []
    for _ in range(steps):
        total = 0.0
        for w in range(workers):
            words, targets = text(n, vocab, g)
            total += float(model.forward(words, targets).sum() / (targets >= 0).sum())
            model.backward(*views(grad))
            swap.send(w, grad)
        swap.average(mean)
        table_grad, weight_grad = views(mean)
        model.table.sub_(table_grad, alpha=lr)
        sidco.sidco_muon_step(weight_grad, momentum, model.weight, lr=0.02)
        losses.append(total / workers)
    return {"losses": losses, "bytes": swap.bytes, "gradient_bytes": 4 * d}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    for exchange in ("4bit", "sparse"):
        r = train(exchange, a.workers, a.steps)
        shown = ", ".join("%.4f" % r["losses"][i] for i in sorted({0, a.steps // 4, a.steps // 2, a.steps - 1}))
        print(f"{exchange}: loss {shown}; {r['bytes']:.0f} of {r['gradient_bytes']} bytes a worker and step", flush=True)


if __name__ == "__main__":
    main()
