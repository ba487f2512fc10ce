"""Performance cases of the dense operators beside the sparsifier: 4-bit microscaled gradients and products, and the
orthogonalised update.

Each pass makes the calls that one data-parallel worker makes of one of them:
  exchange    the gradient, with the carried residual, becomes blocks of 4-bit codes (error feedback: what the codes do
              not hold stays in the residual); all workers' blocks are then read back and averaged
  roundtrip   a matrix is quantised along its rows and along its columns, as a layer keeps its input until the backward
              pass needs it, and both forms are read back
  infer       a few rows times a weight matrix that was laid out in 4 bits once
  train       a linear layer's step: input, weight and output gradient are quantised, and the three products give the
              output, the input's gradient and the weight's
  orthogonal  a batch of matrices, each brought near the closest one with orthonormal rows or columns by Newton-Schulz products
  update      momentum, its orthogonalisation, and the weights' update with it

A 4-bit block is 32 neighbours of a row: one sign, two exponent and one mantissa bit each (0, 0.5, 1, 1.5, 2, 3, 4, 6),
to nearest, ties to even, over a common power of two, 2^(floor(log2(largest magnitude)) - 2) held as an exponent of 8 bits.
A block that holds an infinity or a NaN has the exponent 255 and stands for NaN.  Rows are padded with zeros to 256.

A case is a dict of plain values:
  entry   one of the above                         dtype   element type of gradient, matrix, input and weight
  d, workers            exchange: length of the flat gradient, number of payloads averaged
  rows, cols, batch     roundtrip, orthogonal and update: the matrix, and how many of them
  rows, inputs, outputs infer and train: the layer
  wide                  infer: the result is kept in 32 bits
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK, PAD = 32, 256
STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LEARNING_RATE, MOMENTUM, WEIGHT_DECAY = 0.02, 0.95, 0.01


def listed():
    return [
        # ResNet-20, the smallest whole model, between four workers: launches and latency
        dict(name="resnet20_exchange", entry="exchange", d=269_722, workers=4, dtype="f32"),
        # VGG19, the largest model, mixed-precision gradients, a node of eight workers
        dict(name="vgg19_exchange_bf16", entry="exchange", d=138_357_544, workers=8, dtype="bf16"),
        # the LSTM's hidden states of one batch (20 sequences of 35 steps): rows that do not fill their last block
        dict(name="lstm_states_roundtrip", entry="roundtrip", rows=700, cols=1500, dtype="f32"),
        # a large batch of a wide layer's inputs
        dict(name="wide_inputs_roundtrip", entry="roundtrip", rows=16_384, cols=4096, dtype="bf16"),
        # VGG's second dense layer for one image
        dict(name="vgg_fc7_one_row", entry="infer", rows=1, inputs=4096, outputs=4096, dtype="bf16", wide=False),
        # the LSTM's decoder over its 10000 words, one step of 20 sequences, logits kept in 32 bits
        dict(name="lstm_decoder_20_rows", entry="infer", rows=20, inputs=1500, outputs=10_000, dtype="f16", wide=True),
        # the LSTM's four gates over one batch
        dict(name="lstm_gates_train", entry="train", rows=700, inputs=1500, outputs=6000, dtype="f32"),
        # VGG's first dense layer, the largest matrix of the models, a large batch
        dict(name="vgg_fc6_train", entry="train", rows=4096, inputs=25_088, outputs=4096, dtype="bf16"),
        # ResNet-50's three smallest 3x3 convolutions as matrices
        dict(name="resnet50_conv2_update", entry="update", batch=3, rows=64, cols=576, dtype="f32"),
        # ResNet-50's six 3x3 convolutions of the fourth group, the products alone, in mixed precision
        dict(name="resnet50_conv4_orthogonal", entry="orthogonal", batch=6, rows=256, cols=2304, dtype="bf16"),
        # the LSTM's four gate matrices, tall, weights in 32 bits
        dict(name="lstm_gates_update", entry="update", batch=4, rows=6000, cols=1500, dtype="f32"),
        # VGG's first dense layer, weights in 16 bits
        dict(name="vgg_fc6_update", entry="update", batch=1, rows=4096, cols=25_088, dtype="bf16"),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; odd, or a round hundred where that is near."""
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    if n >= 1000 and rng.random() < 0.5:
        return n // 100 * 100
    return min(hi, n | 1) if n > 1 else n


def draw(rng):
    """One more case of the ranges of the listed ones."""
    entry = rng.choice(["exchange", "roundtrip", "infer", "train", "orthogonal", "update"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if entry == "exchange":
        return dict(entry=entry, d=_size(rng, 20_000, 138_357_544), workers=rng.randint(1, 8), dtype=dtype)
    if entry == "roundtrip":
        return dict(entry=entry, rows=_size(rng, 16, 16_384), cols=_size(rng, 64, 4096), dtype=dtype)
    if entry == "infer":
        return dict(entry=entry, rows=_size(rng, 1, 48), inputs=_size(rng, 100, 16_384), outputs=_size(rng, 100, 16_384), dtype=dtype,
                    wide=rng.random() < 0.5)
    if entry == "train":
        return dict(entry=entry, rows=_size(rng, 16, 4096), inputs=_size(rng, 64, 8192), outputs=_size(rng, 64, 8192), dtype=dtype)
    rows, cols = _size(rng, 16, 6000), _size(rng, 16, 6000)
    if entry == "update" and dtype == "f16":  # weights of 16 bits are bf16 ones
        dtype = "bf16"
    return dict(entry=entry, batch=rng.randint(1, max(1, min(6, 24_000_000 // (rows * cols)))), rows=rows, cols=cols, dtype=dtype)


def _up(n, m):
    return -(-n // m) * m


# ---- the 4-bit format in 32 bits ------------------------------------------------------------------------------------


def _quantize(x):
    """Rows of float32 -> (values without their scale, exponent codes), padded to PAD columns."""
    rows, cols = x.shape
    blocks = torch.nn.functional.pad(x, (0, _up(cols, PAD) - cols)).view(rows, -1, BLOCK)
    top = blocks.abs().amax(-1, keepdim=True)
    exponent = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(min=-127)
    bad = ~torch.isfinite(top)
    exponent = torch.where(bad, 128, exponent)
    small = torch.ldexp(blocks, torch.where(bad, 0, -exponent))
    size = small.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    value = torch.copysign((torch.round(size / step) * step).clamp(max=6.0), small)
    return torch.where(bad, 0.0, value), exponent + 127


def _values(value, code):
    """What (values without their scale, exponent codes) stand for, padding included."""
    x = torch.ldexp(value, code - 127)
    return torch.where(code == 255, math.nan, x).view(x.shape[0], -1)


def _rounded(x):
    """A float32 matrix as its 4-bit blocks stand for it."""
    return _values(*_quantize(x))[:, : x.shape[1]]


def _pack(value, code):
    size = value.abs()
    number = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8)
    nibble = (number | (torch.signbit(value).to(torch.uint8) << 3)).view(value.shape[0], -1)
    return (nibble[:, 0::2] | (nibble[:, 1::2] << 4)).contiguous(), code.to(torch.uint8).view(value.shape[0], -1).contiguous()


def _unpack(codes, scales, cols):
    """Packed rows as the float32 values that they stand for."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32, device=codes.device)
    table = torch.cat([table, -table])
    value = table[torch.stack([codes & 15, codes >> 4], -1).int()]
    return _values(value.view(codes.shape[0], -1, BLOCK), scales.int()[:, :, None])[:, :cols]


# ---- the inputs -----------------------------------------------------------------------------------------------------


def _laplace(g, *shape, width=1e-3):
    u = torch.rand(*shape, generator=g, device="cuda") - 0.5
    return -width * torch.sign(u) * torch.log1p(-2 * u.abs().clamp(max=0.4999999))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPES[case["dtype"]]
    s = dict(case=case, entry=case["entry"])
    empty = lambda *shape, dtype=t: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    bytes_of = lambda rows, cols: (empty(rows, _up(cols, PAD) // 2, dtype=torch.uint8), empty(rows, _up(cols, PAD) // BLOCK, dtype=torch.uint8))  # noqa: E731
    if s["entry"] == "exchange":
        d = case["d"]
        s["grad"] = _laplace(g, d).to(t)
        s["residual"] = _laplace(g, d, width=1e-4)
        s["codes"], s["scales"] = bytes_of(case["workers"], d)
        for w in range(1, case["workers"]):  # what the others have sent; the first place is this worker's
            c, e = _pack(*_quantize(_laplace(g, 1, d)))
            s["codes"][w], s["scales"][w] = c[0], e[0]
        s["dense"] = empty(d, dtype=torch.float32)
        return s
    shape = (case.get("batch"), case["rows"], case.get("cols"))
    if s["entry"] == "orthogonal":
        s["x"] = (normal(*shape) * 1e-3).to(t)
        s["out"] = empty(*shape)
        return s
    if s["entry"] == "update":
        s["grad"] = (normal(*shape) * 1e-3).to(t)
        s["momentum"] = normal(*shape) * 1e-2
        s["weight"] = (normal(*shape) / math.sqrt(case["cols"])).to(t)
        return s
    rows = case["rows"]
    if s["entry"] == "roundtrip":
        cols = case["cols"]
        x = normal(rows, cols) * torch.exp(normal(1, cols))  # features of different scale
        s["x"] = x.to(t)
        s["along_rows"], s["along_cols"] = bytes_of(rows, cols), bytes_of(cols, rows)
        s["out"], s["out_t"] = empty(rows, cols, dtype=torch.bfloat16), empty(cols, rows, dtype=torch.bfloat16)
        return s
    n, m = case["inputs"], case["outputs"]
    s["x"] = (normal(rows, n) * torch.exp(0.5 * normal(1, n))).to(t)
    w = normal(m, n) / math.sqrt(n)
    if s["entry"] == "infer":
        s["weight"] = _pack(*_quantize(w))
        s["y"] = empty(rows, m, dtype=torch.float32 if case["wide"] else t)
        return s
    s["weight"], s["dy"] = w.to(t), (normal(rows, m) * 1e-3).to(t)
    s["forms"] = {k: (bytes_of(a, b), bytes_of(b, a)) for k, a, b in (("x", rows, n), ("weight", m, n), ("dy", rows, m))}
    s["y"], s["dx"], s["dw"] = empty(rows, m), empty(rows, n), empty(m, n, dtype=torch.float32)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(state):
    return (_run_own if own else _run_plain)(state)


def _learning_scale(case):
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def _run_own(s):
    import paper_2101_10761_amd as sidco

    case = s["case"]
    if s["entry"] == "exchange":
        sidco.sidco_mx4_compress(s["grad"], s["residual"], s["codes"][0], s["scales"][0])
        sidco.sidco_mx4_aggregate(s["codes"], s["scales"], s["dense"], scale=1.0 / case["workers"])
        return {"dense": s["dense"], "residual": s["residual"]}
    if s["entry"] == "orthogonal":
        sidco.sidco_orthogonalize(s["x"], s["out"], steps=STEPS, coef=COEF, eps=EPS)
        return {"out": s["out"]}
    if s["entry"] == "update":
        sidco.sidco_muon_step(s["grad"], s["momentum"], s["weight"], lr=LEARNING_RATE, mu=MOMENTUM, weight_decay=WEIGHT_DECAY,
                              scale=_learning_scale(case), steps=STEPS, coef=COEF, eps=EPS)
        return {"weight": s["weight"], "momentum": s["momentum"]}
    if s["entry"] == "roundtrip":
        a, b = s["along_rows"], s["along_cols"]
        sidco.sidco_mx4_quantize(s["x"], a[0], a[1], b[0], b[1])
        sidco.sidco_mx4_dequantize(a[0], a[1], s["out"])
        sidco.sidco_mx4_dequantize(b[0], b[1], s["out_t"])
        return {"out": s["out"], "out_t": s["out_t"]}
    if s["entry"] == "infer":
        sidco.sidco_mx4_linear(s["x"], s["weight"][0], s["weight"][1], s["y"])
        return {"y": s["y"]}
    (xr, xc), (wr, wc), (gr, gc) = (s["forms"][k] for k in ("x", "weight", "dy"))
    rows, n, m = case["rows"], case["inputs"], case["outputs"]
    sidco.sidco_mx4_quantize(s["x"], xr[0], xr[1], xc[0], xc[1])
    sidco.sidco_mx4_quantize(s["weight"], wr[0], wr[1], wc[0], wc[1])
    sidco.sidco_mx4_matmul(xr[0], xr[1], wr[0], wr[1], n, s["y"])
    sidco.sidco_mx4_quantize(s["dy"], gr[0], gr[1], gc[0], gc[1])
    sidco.sidco_mx4_matmul(gr[0], gr[1], wc[0], wc[1], m, s["dx"])
    sidco.sidco_mx4_matmul(gc[0], gc[1], xc[0], xc[1], rows, s["dw"])
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


def _orthogonal_plain(x):
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = COEF
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _run_plain(s):
    case = s["case"]
    if s["entry"] == "exchange":
        d, workers = case["d"], case["workers"]
        acc = s["grad"].float() + s["residual"]
        mine = _rounded(acc[None])[0]
        s["residual"].copy_(torch.where(torch.isfinite(mine), acc - mine, acc))
        total = mine
        if workers > 1:
            total = total + _unpack(s["codes"][1:], s["scales"][1:], d).sum(0)
        s["dense"].copy_(total / workers)
        return {"dense": s["dense"], "residual": s["residual"]}
    if s["entry"] == "orthogonal":
        s["out"].copy_(_orthogonal_plain(s["x"].float()))
        return {"out": s["out"]}
    if s["entry"] == "update":
        g, m, w = s["grad"].float(), s["momentum"], s["weight"]
        m.mul_(MOMENTUM).add_(g)
        x = _orthogonal_plain(g + MOMENTUM * m)
        w.copy_(w.float() * (1 - LEARNING_RATE * WEIGHT_DECAY) - (LEARNING_RATE * _learning_scale(case)) * x)
        return {"weight": w, "momentum": m}
    if s["entry"] == "roundtrip":
        x = s["x"].float()
        s["out"].copy_(_rounded(x))
        s["out_t"].copy_(_rounded(x.t()))
        return {"out": s["out"], "out_t": s["out_t"]}
    x = s["x"].float()
    if s["entry"] == "infer":
        s["y"].copy_(_rounded(x) @ _unpack(*s["weight"], case["inputs"]).t())
        return {"y": s["y"]}
    w, dy = s["weight"].float(), s["dy"].float()
    s["y"].copy_(_rounded(x) @ _rounded(w).t())
    s["dx"].copy_(_rounded(dy) @ _rounded(w.t()).t())
    s["dw"].copy_(_rounded(dy.t()) @ _rounded(x.t()).t())
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

_SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_blocks(x):
    """Rows in 64 bits as their blocks stand for them: each magnitude goes up past every midpoint that it lies above, and at
    one from an odd number to the even one."""
    rows, cols = x.shape
    x = torch.cat([x, x.new_zeros(rows, -cols % BLOCK)], 1).view(rows, -1, BLOCK)
    top = x.abs().max(-1, keepdim=True).values
    scale = ((top.view(torch.int64) >> 52) - 2 << 52).view(torch.float64)  # the power of two at or below, over four
    scale = torch.where(top > 2.0**-125, scale, 2.0**-127)
    size, value = x.abs() / scale, torch.zeros_like(x)
    for k in range(7):
        middle, jump = (_SIZES[k] + _SIZES[k + 1]) / 2, _SIZES[k + 1] - _SIZES[k]
        value += jump * ((size > middle) | ((size == middle) & (k % 2 == 1)))
    value = torch.where(torch.isfinite(top), torch.sign(x) * value * scale, math.nan)
    return value.view(rows, -1)[:, :cols]


def _exact_packed(codes, scales, cols):
    nibble = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    for k in (0, 1):
        number = (codes >> (4 * k)) & 7
        value = sum(size * (number == i) for i, size in enumerate(_SIZES))
        nibble[:, k::2] = value.double() * (1 - 2 * ((codes >> (4 * k)) >> 3 & 1).double())
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=codes.device), scales.double() - 127)
    return (nibble * power.repeat_interleave(BLOCK, 1))[:, :cols]


def _exact_orthogonal(x):
    tall = x.shape[1] > x.shape[2]  # odd polynomials of a matrix and of its transpose are each other's transpose
    x = x.mT.contiguous() if tall else x
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS)
    a, b, c = COEF
    for _ in range(STEPS):
        xt = x.mT.contiguous()
        y = torch.matmul(torch.matmul(x, xt), x)
        x, y = a * x + b * y, torch.matmul(torch.matmul(x, xt), y)
        x = x + c * y
    return x.mT if tall else x


def exact(case, seed):
    s = prepare(case, seed)
    if s["entry"] == "exchange":
        acc = (s["grad"].float() + s["residual"]).double()  # the accumulated vector is a 32-bit one by definition
        mine = _exact_blocks(acc[None])[0]
        total = mine.clone()
        for w in range(1, case["workers"]):
            total += _exact_packed(s["codes"][w : w + 1], s["scales"][w : w + 1], case["d"])[0]
        return {"dense": total / case["workers"], "residual": acc - mine}
    if s["entry"] == "orthogonal":
        return {"out": _exact_orthogonal(s["x"].double())}
    if s["entry"] == "update":
        g, w = s["grad"].double(), s["weight"].double()
        m = MOMENTUM * s["momentum"].double() + g
        x = _exact_orthogonal(g + MOMENTUM * m)
        return {"weight": (1 - LEARNING_RATE * WEIGHT_DECAY) * w - LEARNING_RATE * _learning_scale(case) * x, "momentum": m}
    x = s["x"].double()
    if s["entry"] == "roundtrip":
        return {"out": _exact_blocks(x), "out_t": _exact_blocks(x.t().contiguous())}
    if s["entry"] == "infer":
        return {"y": _exact_blocks(x) @ _exact_packed(*s["weight"], case["inputs"]).t()}
    w, dy = s["weight"].double(), s["dy"].double()
    dw = _exact_blocks(dy.t().contiguous()) @ _exact_blocks(x.t().contiguous()).t()
    return {"y": _exact_blocks(x) @ _exact_blocks(w).t(), "dx": _exact_blocks(dy) @ _exact_blocks(w.t().contiguous()).t(), "dw": dw}


def work(case):
    """Bytes with each input read and each output written once, and operations (symmetric products count half)."""
    b = 4 if case["dtype"] == "f32" else 2
    packed = 17 / 32  # a code and its share of the exponent, bytes an element
    if case["entry"] == "exchange":
        d, w = case["d"], case["workers"]
        return {"bytes": d * (b + 8 + packed + w * packed + 4), "flops": d * (8 + 2 * w)}
    if case["entry"] == "roundtrip":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (b + 4 * packed + 4), "flops": 16 * n}
    if case["entry"] in ("orthogonal", "update"):
        m, n = sorted((case["rows"], case["cols"]))
        each = 2 * b if case["entry"] == "orthogonal" else b + 8 + 2 * b
        return {"bytes": case["batch"] * m * n * each, "flops": case["batch"] * STEPS * (3 * m * m * n + m**3)}
    r, n, m = case["rows"], case["inputs"], case["outputs"]
    if case["entry"] == "infer":
        return {"bytes": r * n * b + n * m * packed + r * m * (4 if case["wide"] else b), "flops": 2 * r * n * m}
    return {"bytes": b * 2 * (r * n + r * m) + n * m * (b + 4), "flops": 6 * r * n * m}
