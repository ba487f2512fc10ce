"""Performance cases of a language model's operators beside the dense ones: the embedding and its gradient, dropout, and
softmax cross entropy over a vocabulary.

Each pass makes the calls that one data-parallel worker makes of one of them:
  lookup       tokens become rows of the table, times a scale
  lookup_grad  the rows' gradient becomes the table's, added up for each token (accumulate: on top of what is there, as
               with a table that is the decoder's weight too)
  dropout      elements are kept by a counter-based generator's numbers and rescaled, (add) and a residual is added
  score        hidden rows and the decoder's weight become each row's loss and the logarithm of its sum of exponentials
  train        the same, and the gradients of hidden rows and weight for given gradients of the losses

A token or target outside the vocabulary stands for padding: its row is zeros, it has no loss and no gradient.

The generator: block b of a sequence is Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) of the counter b with the seed as
its key, eight numbers of 16 bits, low halves first; a row of c elements takes ceil(c / 8) blocks.  An element is kept where
its number is at least T = floor(65536 p + 1/2), and is then times 65536 / (65536 - T).

A case is a dict of plain values:
  entry    one of the above                    dtype    element type of table, rows, hidden rows and weight
  n        tokens or rows                      out      element type of the table's or the weight's gradient
  dim      a row's elements                    index    element type of tokens and targets
  vocab    rows of table and weight            padding  share of tokens or targets that are padding
  scale    of the lookup                       p        of the dropout
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
INDEX = {"i32": torch.int32, "i64": torch.int64}
M32 = 0xFFFFFFFF


def listed():
    return [
        # the LSTM's batch, 20 sequences of 35 words out of 10000: launches and latency
        dict(name="lstm_lookup", entry="lookup", n=700, dim=1500, vocab=10_000, dtype="f32", index="i64", scale=1.0, padding=0.0),
        # a long batch of a wide model in mixed precision, rows scaled by the root of their length
        dict(name="wide_lookup_bf16", entry="lookup", n=65_536, dim=4096, vocab=131_072, dtype="bf16", index="i32", scale=64.0, padding=0.0),
        # the LSTM's table gradient, whole, as the sparsifier takes it
        dict(name="lstm_lookup_grad", entry="lookup_grad", n=700, dim=1500, vocab=10_000, dtype="f32", out="f32", index="i64", scale=1.0,
             padding=0.0, accumulate=False),
        # a padded batch of odd sizes added to the decoder's gradient, everything in half precision
        dict(name="tied_lookup_grad_f16", entry="lookup_grad", n=4099, dim=1111, vocab=49_999, dtype="f16", out="f16", index="i64", scale=1.0,
             padding=0.07, accumulate=True),
        # the long batch's table gradient in 32 bits
        dict(name="wide_lookup_grad", entry="lookup_grad", n=65_536, dim=4096, vocab=131_072, dtype="bf16", out="f32", index="i32", scale=64.0,
             padding=0.0, accumulate=False),
        # between the LSTM's layers
        dict(name="lstm_dropout", entry="dropout", n=700, dim=1500, dtype="f32", p=0.5, add=False),
        # a wide model's block output with the residual
        dict(name="wide_dropout_add", entry="dropout", n=65_536, dim=4096, dtype="bf16", p=0.1, add=True),
        # the LSTM's next word, one step of 20 sequences
        dict(name="lstm_score_20_rows", entry="score", n=20, dim=1500, vocab=10_000, dtype="f32", index="i64", padding=0.0),
        # a single token of a wide model
        dict(name="wide_score_one_row", entry="score", n=1, dim=4096, vocab=131_072, dtype="bf16", index="i64", padding=0.0),
        # the LSTM's batch
        dict(name="lstm_train", entry="train", n=700, dim=1500, vocab=10_000, dtype="f32", out="f32", index="i64", padding=0.0,
             accumulate=False),
        # a padded micro-batch in half precision, the weight's gradient added up in 32 bits over several of them
        dict(name="micro_batch_train_f16", entry="train", n=2049, dim=1024, vocab=49_999, dtype="f16", out="f32", index="i64", padding=0.07,
             accumulate=True),
        # a wide model's batch in mixed precision
        dict(name="wide_train_bf16", entry="train", n=8192, dim=4096, vocab=131_072, dtype="bf16", out="bf16", index="i64", padding=0.03,
             accumulate=False),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; odd, or a multiple of 128 where there is room for one."""
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    if n >= 256 and rng.random() < 0.5:
        return n // 128 * 128
    return min(hi, n | 1) if n > 1 else n


def draw(rng):
    """One more case of the ranges of the listed ones."""
    entry = rng.choice(["lookup", "lookup_grad", "dropout", "score", "train"])
    dtype, index = rng.choice(["f32", "bf16", "f16"]), rng.choice(["i32", "i64"])
    padding = rng.choice([0.0, 0.03, 0.3])
    if entry == "dropout":
        return dict(entry=entry, n=_size(rng, 1, 32_768), dim=_size(rng, 64, 4096), dtype=dtype, p=rng.choice([0.1, 0.25, 0.5, 0.65]),
                    add=rng.random() < 0.5)
    vocab = _size(rng, 500, 131_072)
    if entry in ("lookup", "lookup_grad"):
        case = dict(entry=entry, n=_size(rng, 1, 32_768), dim=_size(rng, 64, 4096), vocab=vocab, dtype=dtype, index=index,
                    scale=rng.choice([1.0, 22.5, 64.0]), padding=padding)
        return case if entry == "lookup" else dict(case, out=rng.choice(["f32", dtype]), accumulate=rng.random() < 0.5)
    case = dict(entry=entry, dim=_size(rng, 64, 4096), vocab=vocab, dtype=dtype, index=index, padding=padding)
    if entry == "score":
        return dict(case, n=_size(rng, 1, 48) if rng.random() < 0.5 else _size(rng, 48, 4096))
    # operands in 32 bits cost several times those of 16
    return dict(case, n=_size(rng, 16, 8192 if dtype != "f32" else 2048), out=rng.choice(["f32", dtype]), accumulate=rng.random() < 0.5)


# ---- the inputs -----------------------------------------------------------------------------------------------------


def _words(g, case):
    """Words as a text has them, the k-th most frequent about 1 / k as often, some of them padding."""
    n, vocab = case["n"], case["vocab"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    words = (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)
    hidden = torch.rand(n, generator=g, device="cuda") < case["padding"]
    return torch.where(hidden, -100, words).to(INDEX[case["index"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, n, dim = DTYPES[case["dtype"]], case["n"], case["dim"]
    s = dict(case=case, entry=case["entry"])
    empty = lambda *shape, dtype=t: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    if s["entry"] == "dropout":
        s["seed"], s["offset"] = (0x9E3779B97F4A7C15 * (seed + 1)) & 0x7FFFFFFFFFFFFFFF, 1_000_003 * (seed % 1000)
        s["x"], s["y"] = normal(n, dim).to(t), empty(n, dim)
        s["residual"] = normal(n, dim).to(t) if case["add"] else None
        return s
    vocab = case["vocab"]
    s["words"] = _words(g, case)
    if s["entry"] == "lookup":
        s["table"] = (normal(vocab, dim) / math.sqrt(dim)).to(t)
        s["rows"] = empty(n, dim)
        return s
    if s["entry"] == "lookup_grad":
        s["grad"] = (normal(n, dim) * (1e-2 if case["dtype"] == "f16" else 1e-4)).to(t)
        o = DTYPES[case["out"]]
        s["table_grad"] = (normal(vocab, dim) * 1e-2).to(o) if case["accumulate"] else empty(vocab, dim, dtype=o)
        return s
    # hidden rows of about unit variance that know their target, some better than others
    w = normal(vocab, dim) / math.sqrt(dim)
    target = s["words"].clamp(min=0).long()
    s["x"] = (normal(n, dim) + w[target] * (math.log(vocab) * 1.5 * torch.rand(n, 1, generator=g, device="cuda"))).to(t)
    s["weight"] = w.to(t)
    s["loss"], s["lse"] = empty(n, dtype=torch.float32), empty(n, dtype=torch.float32)
    if s["entry"] == "train":
        o = DTYPES[case["out"]]
        # the mean over the targets, in half precision times a loss scale
        s["loss_grad"] = torch.full((n,), (4096.0 if case["dtype"] == "f16" else 1.0) / n, device="cuda")
        s["x_grad"] = empty(n, dim)
        before = 1e-2 if case["dtype"] == "f16" else 1e-4
        s["weight_grad"] = normal(vocab, dim).mul_(before).to(o) if case["accumulate"] else empty(vocab, dim, dtype=o)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2101_10761_amd as sidco

    case = s["case"]
    if s["entry"] == "lookup":
        sidco.sidco_embedding(s["table"], s["words"], s["rows"], scale=case["scale"])
        return {"rows": s["rows"]}
    if s["entry"] == "lookup_grad":
        sidco.sidco_embedding_grad(s["grad"], s["words"], s["table_grad"], scale=case["scale"], accumulate=case["accumulate"])
        return {"table_grad": s["table_grad"]}
    if s["entry"] == "dropout":
        sidco.sidco_dropout(s["x"], s["y"], case["p"], s["seed"], offset=s["offset"], residual=s["residual"])
        return {"y": s["y"]}
    sidco.sidco_cross_entropy(s["x"], s["weight"], s["words"], s["loss"], s["lse"])
    if s["entry"] == "score":
        return {"loss": s["loss"], "lse": s["lse"]}
    sidco.sidco_cross_entropy_grad(s["x"], s["weight"], s["words"], s["lse"], s["loss_grad"], s["x_grad"], s["weight_grad"],
                                   accumulate=case["accumulate"])
    return {"loss": s["loss"], "lse": s["lse"], "x_grad": s["x_grad"], "weight_grad": s["weight_grad"]}


def _numbers(n, dim, seed, offset):
    """The generator's 16-bit numbers of n rows, products of 32 bits by 32 in 64."""
    per_row = -(-dim // 8)
    block = torch.arange(offset, offset + n * per_row, device="cuda")
    c0, c1 = block & M32, block >> 32
    c2 = c3 = torch.zeros_like(block)
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & M32) ^ c1 ^ k0, b & M32, ((a >> 32) & M32) ^ c3 ^ k1, a & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).view(n, per_row * 8)[:, :dim]


def _run_plain(s):
    case, entry = s["case"], s["entry"]
    if entry == "dropout":
        threshold = math.floor(65536 * case["p"] + 0.5)
        kept = _numbers(case["n"], case["dim"], s["seed"], s["offset"]) >= threshold
        y = torch.where(kept, s["x"].float() * (65536 / (65536 - threshold)), 0.0)
        s["y"].copy_(y + s["residual"].float() if case["add"] else y)
        return {"y": s["y"]}
    words = s["words"].long()
    inside = (words >= 0) & (words < case["vocab"])
    word = torch.where(inside, words, 0)
    if entry == "lookup":
        s["rows"].copy_(torch.where(inside[:, None], s["table"][word].float() * case["scale"], 0.0))
        return {"rows": s["rows"]}
    if entry == "lookup_grad":
        total = torch.zeros(case["vocab"], case["dim"], device="cuda")
        total.index_add_(0, word, torch.where(inside[:, None], s["grad"].float() * case["scale"], 0.0))
        s["table_grad"].copy_(total + s["table_grad"].float() if case["accumulate"] else total)
        return {"table_grad": s["table_grad"]}
    x, w = s["x"].float(), s["weight"].float()
    logits = x @ w.t()
    top = logits.max(1, keepdim=True).values
    p = torch.exp(logits - top)
    total = p.sum(1, keepdim=True)
    s["lse"].copy_((top + torch.log(total))[:, 0])
    s["loss"].copy_(torch.where(inside, s["lse"] - logits.gather(1, word[:, None])[:, 0], 0.0))
    if entry == "score":
        return {"loss": s["loss"], "lse": s["lse"]}
    p = p / total
    p[torch.arange(case["n"], device="cuda"), word] -= 1
    p = torch.where(inside[:, None], p * s["loss_grad"][:, None], 0.0)
    s["x_grad"].copy_(p @ w)
    weight_grad = p.t() @ x
    s["weight_grad"].copy_(weight_grad + s["weight_grad"].float() if case["accumulate"] else weight_grad)
    return {"loss": s["loss"], "lse": s["lse"], "x_grad": s["x_grad"], "weight_grad": s["weight_grad"]}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def _exact_kept(n, dim, seed, offset, threshold):
    """The generator with its words in halves of 16 bits, so that no product leaves 48 bits."""

    def times(word, by):
        low, high = word * (by & 0xFFFF), word * (by >> 16)
        total = low + ((high & 0xFFFF) << 16)
        return (high >> 16) + (total >> 32), total & M32

    per_row = (dim + 7) // 8
    rows = torch.arange(n, device="cuda")[:, None] * per_row + torch.arange(per_row, device="cuda")[None] + offset
    state = [rows % 2**32, rows // 2**32, torch.zeros_like(rows), torch.zeros_like(rows)]
    for r in range(10):
        k0, k1 = (seed % 2**32 + r * 0x9E3779B9) % 2**32, (seed // 2**32 + r * 0xBB67AE85) % 2**32
        (ah, al), (bh, bl) = times(state[0], 0xD2511F53), times(state[2], 0xCD9E8D57)
        state = [bh ^ state[1] ^ k0, bl, ah ^ state[3] ^ k1, al]
    kept = torch.empty(n, per_row, 8, dtype=torch.bool, device="cuda")
    for i in range(8):
        kept[:, :, i] = (state[i // 2] // (65536 if i % 2 else 1)) % 65536 >= threshold
    return kept.view(n, -1)[:, :dim]


def exact(case, seed):
    s = prepare(case, seed)
    n, dim = case["n"], case["dim"]
    if s["entry"] == "dropout":
        threshold = int(65536 * case["p"] + 0.5)
        kept = _exact_kept(n, dim, s["seed"], s["offset"], threshold)
        y = s["x"].double() * kept * 65536 / (65536 - threshold)
        return {"y": y + s["residual"].double() if case["add"] else y}
    vocab, words = case["vocab"], s["words"].long()
    at = ((words >= 0) & (words < vocab)).nonzero()[:, 0]  # places that are no padding
    word = words[at]
    if s["entry"] == "lookup":
        rows = torch.zeros(n, dim, dtype=torch.float64, device="cuda")
        rows[at] = torch.index_select(s["table"], 0, word).double() * case["scale"]
        return {"rows": rows}
    if s["entry"] == "lookup_grad":
        # running sums of the rows in the order of their words, and what they grow by from word to word
        order = torch.argsort(word, stable=True)
        total = s["table_grad"].double() if case["accumulate"] else torch.zeros(vocab, dim, dtype=torch.float64, device="cuda")
        if len(at):
            present, count = torch.unique_consecutive(word[order], return_counts=True)
            ends = torch.cumsum(count, 0) - 1
            for c in range(0, dim, 512):
                run_sum = torch.cumsum(s["grad"][at[order], c : c + 512].double() * case["scale"], 0)[ends]
                total[present, c : c + 512] += torch.diff(run_sum, dim=0, prepend=run_sum.new_zeros(1, run_sum.shape[1]))
        return {"table_grad": total}
    x, w = s["x"].double(), s["weight"].double()
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    train = s["entry"] == "train"
    if train:
        dx, dw = torch.zeros_like(x), s["weight_grad"].double() if case["accumulate"] else torch.zeros_like(w)
        g = torch.zeros(n, dtype=torch.float64, device="cuda")
        g[at] = s["loss_grad"][at].double()
    wt = w.t().contiguous()
    for r in range(0, n, 1024):  # some rows at a time
        rows = slice(r, min(n, r + 1024))
        logits = torch.matmul(x[rows], wt)
        lse[rows] = torch.logsumexp(logits, 1)
        here = (at >= rows.start) & (at < rows.stop)
        i, v = at[here] - r, word[here]
        loss[at[here]] = lse[at[here]] - logits[i, v]
        if train:
            logits.sub_(lse[rows, None]).exp_()
            logits[i, v] -= 1.0
            logits.mul_(g[rows, None])
            dx[rows] = torch.matmul(logits, w)
            dw += torch.matmul(logits.t().contiguous(), x[rows])
    return {"loss": loss, "lse": lse, **({"x_grad": dx, "weight_grad": dw} if train else {})}


def _distinct(n, vocab):
    """How many different words n of _words have, on average."""
    k = np.arange(1, vocab + 1)
    return float(-np.expm1(n * np.log1p(-np.log1p(1 / k) / math.log(vocab + 1))).sum())


def work(case):
    """Bytes with each input read once and each output written once, and operations.  The gradient's three products are counted
    once each; that the logits are not kept, and formed twice for it, is not."""
    size = {"f32": 4, "f16": 2, "bf16": 2, "i32": 4, "i64": 8}
    n, dim, b = case["n"], case["dim"], size[case["dtype"]]
    if case["entry"] == "dropout":
        return {"bytes": n * dim * b * (3 if case["add"] else 2), "flops": n * dim * (2 if case["add"] else 1)}
    vocab, index = case["vocab"], n * size[case["index"]]
    if case["entry"] == "lookup":
        return {"bytes": int((_distinct(n, vocab) + n) * dim * b) + index, "flops": n * dim}
    if case["entry"] == "lookup_grad":
        table = 2 * _distinct(n, vocab) if case["accumulate"] else vocab
        return {"bytes": int(n * dim * b + table * dim * size[case["out"]]) + index, "flops": 2 * n * dim}
    if case["entry"] == "score":
        return {"bytes": (n + vocab) * dim * b + index + 8 * n, "flops": 2 * n * dim * vocab}
    weight = size[case["out"]] * (2 if case["accumulate"] else 1)
    return {"bytes": (2 * n + vocab) * dim * b + vocab * dim * weight + index + 12 * n, "flops": 6 * n * dim * vocab}
