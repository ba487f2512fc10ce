"""A training run of a small network whose workers use the dense operators together: `python -m paper_2101_10761_amd.dense_step`.

Every worker's layers multiply in 4 bits, forward and backward (sidco_mx4_quantize, sidco_mx4_matmul).  The flat gradient is
exchanged with error feedback, either dense in 4 bits (sidco_mx4_compress, sidco_mx4_aggregate) or sparse as selected pairs
(sidco_compress, sidco_scatter_add), and the averaged gradient moves the weights through the orthogonalised momentum
(sidco_muon_step).  At the end the weights are laid out once in 4 bits and the network answers single rows (sidco_mx4_linear).

The workers are simulated one after the other on one GPU, each with its own data and residual; what crosses between them is
what a collective would carry.  The task is synthetic: a random two-layer network is the teacher, the loss is the mean square.
"""
from __future__ import annotations

import argparse

from . import binding as sidco


class Packed:
    """A matrix in 4 bits along its rows and, transposed, along its columns."""

    def __init__(self, rows: int, cols: int, device):
        import torch
        empty = lambda n: torch.empty(n, dtype=torch.uint8, device=device)  # noqa: E731
        self.rows = empty(sidco.sidco_mx4_code_bytes(rows, cols)), empty(sidco.sidco_mx4_scale_bytes(rows, cols))
        self.cols = empty(sidco.sidco_mx4_code_bytes(cols, rows)), empty(sidco.sidco_mx4_scale_bytes(cols, rows))

    def take(self, x) -> "Packed":
        sidco.sidco_mx4_quantize(x, *self.rows, *self.cols)
        return self


class Layer:
    """y = x W^T with all three products in 4 bits."""

    def __init__(self, weight, batch: int):
        import torch
        self.outputs, self.inputs = weight.shape
        self.batch, dev = batch, weight.device
        self.w, self.x, self.dy = Packed(*weight.shape, dev), Packed(batch, self.inputs, dev), Packed(batch, self.outputs, dev)
        self.y = torch.empty(batch, self.outputs, device=dev)
        self.dx = torch.empty(batch, self.inputs, device=dev)

    def forward(self, x, weight):
        self.x.take(x)
        self.w.take(weight)
        sidco.sidco_mx4_matmul(*self.x.rows, *self.w.rows, self.inputs, self.y)
        return self.y

    def backward(self, dy, weight_grad):
        """The input's gradient; the weight's is written to weight_grad, a view into the flat gradient."""
        self.dy.take(dy)
        sidco.sidco_mx4_matmul(*self.dy.cols, *self.x.cols, self.batch, weight_grad)
        sidco.sidco_mx4_matmul(*self.dy.rows, *self.w.cols, self.outputs, self.dx)
        return self.dx


class Exchange4Bit:
    """All workers' gradients averaged through 4-bit blocks with error feedback."""

    def __init__(self, workers: int, d: int, device):
        import torch
        self.codes = torch.empty(workers, sidco.sidco_mx4_code_bytes(1, d), dtype=torch.uint8, device=device)
        self.scales = torch.empty(workers, sidco.sidco_mx4_scale_bytes(1, d), dtype=torch.uint8, device=device)
        self.residuals = torch.zeros(workers, d, device=device)

    @property
    def bytes(self) -> float:
        """What one worker sends in a step."""
        return self.codes.shape[1] + self.scales.shape[1]

    def send(self, worker: int, grad) -> None:
        sidco.sidco_mx4_compress(grad, self.residuals[worker], self.codes[worker], self.scales[worker])

    def average(self, out) -> None:
        sidco.sidco_mx4_aggregate(self.codes, self.scales, out, scale=1.0 / len(self.codes))


class ExchangeSparse:
    """All workers' gradients averaged through the pairs that the sparsifier selects."""

    def __init__(self, workers: int, d: int, device, delta: float):
        import torch
        cap = sidco.sidco_out_capacity(d, delta)
        self.delta, self.residuals = delta, torch.zeros(workers, d, device=device)
        self.idx = torch.empty(workers, cap, dtype=torch.int32, device=device)
        self.val = torch.empty(workers, cap, device=device)
        self.count = torch.zeros(workers, dtype=torch.int32, device=device)
        self.eta = torch.zeros(workers, device=device)
        self.pairs, self.sends = torch.zeros(1, dtype=torch.int64, device=device), 0

    @property
    def bytes(self) -> float:
        """What one worker has sent in a step on average: an index and a value for each pair that was selected."""
        return 8 * int(self.pairs) / max(1, self.sends)

    def send(self, worker: int, grad) -> None:
        sidco.sidco_compress(grad, self.residuals[worker], self.delta, sidco.DIST_EXP, 2, self.idx[worker], self.val[worker],
                             self.count[worker:worker + 1], self.eta[worker:worker + 1])
        self.pairs += self.count[worker:worker + 1]
        self.sends += 1

    def average(self, out) -> None:
        out.zero_()
        for w in range(len(self.idx)):
            sidco.sidco_scatter_add(out, self.idx[w], self.val[w], self.count[w:w + 1], 1.0 / len(self.idx))


def train(exchange: str = "4bit", workers: int = 4, steps: int = 60, batch: int = 256, sizes=(384, 512, 96), lr: float = 0.02,
          delta: float = 0.05, seed: int = 0) -> dict:
    """Trains and returns {"losses": [...], "answers": (largest difference of a single row's answer, its size), "bytes": of a worker's
    message, "gradient_bytes": of the gradient in float32}."""
    import torch
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    n, hidden, m = sizes
    teacher = normal(hidden, n) / n ** 0.5, normal(m, hidden) / hidden ** 0.5
    weights = [normal(hidden, n) / n ** 0.5, normal(m, hidden) / hidden ** 0.5]
    shapes = [w.shape for w in weights]
    d = sum(w.numel() for w in weights)
    grad, mean, momentum = (torch.zeros(d, device=dev) for _ in range(3))

    def views(flat):
        out, at = [], 0
        for s in shapes:
            out.append(flat[at:at + s[0] * s[1]].view(s))
            at += s[0] * s[1]
        return out

    layers = [Layer(w, batch) for w in weights]
    swap = Exchange4Bit(workers, d, dev) if exchange == "4bit" else ExchangeSparse(workers, d, dev, delta)
    losses = []
    for step in range(steps):
        total = 0.0
        for w in range(workers):
            x = normal(batch, n)
            want = torch.relu(x @ teacher[0].t()) @ teacher[1].t()
            h = torch.relu(layers[0].forward(x, weights[0]))
            diff = layers[1].forward(h, weights[1]) - want
            total += float(diff.square().mean())
            g0, g1 = views(grad)
            dh = layers[1].backward(diff * (2.0 / diff.numel()), g1)
            layers[0].backward(dh * (h > 0), g0)
            swap.send(w, grad)
        swap.average(mean)
        now = lr * (1 - step / steps)
        for weight, gw, mw in zip(weights, views(mean), views(momentum)):
            sidco.sidco_muon_step(gw, mw, weight, lr=now, scale=max(1.0, weight.shape[0] / weight.shape[1]) ** 0.5)
        losses.append(total / workers)

    # single rows on weights laid out once; the same products on 256 rows are the check
    packed = [Packed(*w.shape, dev).take(w) for w in weights]
    x = normal(batch, n)
    many = layers[1].forward(torch.relu(layers[0].forward(x, weights[0])), weights[1])
    h, y = torch.empty(1, hidden, device=dev), torch.empty(1, m, device=dev)
    worst = 0.0
    for row in (0, batch // 2, batch - 1):
        sidco.sidco_mx4_linear(x[row:row + 1], *packed[0].rows, h)
        sidco.sidco_mx4_linear(torch.relu(h), *packed[1].rows, y)
        worst = max(worst, float((y[0] - many[row]).abs().max()))
    return {"losses": losses, "answers": (worst, float(many.abs().max())), "bytes": swap.bytes, "gradient_bytes": 4 * d}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    for exchange in ("4bit", "sparse"):
        r = train(exchange, a.workers, a.steps)
        shown = ", ".join("%.4f" % r["losses"][i] for i in sorted({0, a.steps // 4, a.steps // 2, a.steps - 1}))
        print(f"{exchange}: loss {shown}; {r['bytes']:.0f} of {r['gradient_bytes']} bytes a worker and step; "
              f"a single row's answer within {r['answers'][0]:.2g} of {r['answers'][1]:.3g}", flush=True)


if __name__ == "__main__":
    main()
