"""GPU: softmax cross entropy over a vocabulary and its gradient against their definition in 64 bits."""
import math

import pytest

import language_reference as ref

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _dtype(t):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[t]


def _case(n, dim, vocab, t, seed=0, padding=0.1, gap=0, wide=True, known=4.0):
    """Rows that know something of their target, a weight, and words, in `gap` more columns than they have."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed * 1009 + n + dim + vocab)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = normal(vocab, dim + gap) / math.sqrt(dim)
    words = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    x = normal(n, dim + gap) + known * torch.rand(n, 1, generator=g, device="cuda") * w[words]
    drop = torch.rand(n, generator=g, device="cuda") < padding
    words = torch.where(drop, torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -100, vocab), words)
    x, w = x.to(_dtype(t)), w.to(_dtype(t))
    at = 1 if gap else 0
    return x[:, at:at + dim], w[:, at:at + dim], words if wide else words.int()


def _near(got, want, off, what):
    torch = _torch()
    miss = (got.double() - want).abs()
    bad = ~(miss <= off)
    assert not bool(bad.any()), (what, int(bad.sum()), float(miss[bad].max()), float(off[bad].min()), bad.nonzero()[:4].tolist())
    # a pair's lost half, a lost column or a missing rounding would hide below sums of worst cases
    size = float(want.norm())
    if want.numel() >= 256 and size > 0:
        # a rounding's own error in the 2-norm is at most half a step, 0.58 of that for values spread evenly
        limit = {torch.float32: 5e-6, torch.float16: 0.7 * 2.0**-11, torch.bfloat16: 0.7 * 2.0**-8}[got.dtype]
        assert float(miss.norm()) <= limit * size, (what, float(miss.norm()) / size)


def _run(x, w, words, g=None, out=None, before=None):
    torch, sidco = _torch(), _sidco()
    n = len(x)
    loss, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    sidco.sidco_cross_entropy(x, w, words, loss, lse)
    dx = torch.full_like(x, 3.0, memory_format=torch.contiguous_format)
    dw = before.clone() if before is not None else torch.full(w.shape, 3.0, dtype=out or w.dtype, device="cuda")
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, dx, dw, accumulate=before is not None)
    torch.cuda.synchronize()
    return loss, lse, dx, dw


SIZES = [(1, 1, 1), (1, 64, 1000), (2, 7, 3), (3, 65, 70), (64, 64, 64), (65, 130, 257), (20, 1500, 700), (257, 96, 1001), (33, 256, 2100), (700, 150, 3000),
         (130, 520, 5000), (5, 8, 20_000)]


@pytest.mark.parametrize("n,dim,vocab", SIZES)
@pytest.mark.parametrize("t,o,accumulate", [("f32", "f32", False), ("f32", "f32", True), ("f16", "f16", False), ("f16", "f32", True), ("bf16", "bf16", True),
                                            ("bf16", "f32", False)])
def test_losses_and_gradients(n, dim, vocab, t, o, accumulate):
    torch = _torch()
    gap = n % 2 * 3
    x, w, words = _case(n, dim, vocab, t, gap=gap, wide=n % 3 > 0)
    g = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)) * (64.0 if t == "f16" else 1.0)
    before = (torch.randn(vocab, dim, device="cuda") * 0.1).to(_dtype(o)) if accumulate else None
    loss, lse, dx, dw = _run(x, w, words, g, _dtype(o), before)
    r = ref.CrossEntropy(x, w, words, g)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")
    _near(dx, *r.x_grad(), "x_grad")
    _near(dw, *r.w_grad(_dtype(o), before), "w_grad")


@pytest.mark.parametrize("n,dim,vocab", [(16, 8, 16), (17, 9, 40), (32, 1024, 33), (33, 100, 700), (40, 1001, 333), (64, 2050, 130), (96, 10, 2000), (97, 64, 300),
                                         (3, 4097, 100), (32, 7, 64), (1, 129, 5000), (31, 4096, 17)])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap", [0, 1, 2])
def test_losses_of_few_rows(n, dim, vocab, t, gap):
    """On both sides of what the kernel for few rows takes, rows that start at any element, steps that are not whole."""
    torch, sidco = _torch(), _sidco()
    x, w, words = _case(n, dim, vocab, t, seed=3, gap=gap)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    sidco.sidco_cross_entropy(x, w, words, loss, lse)
    torch.cuda.synchronize()
    r = ref.CrossEntropy(x, w, words)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_infinite_weights_of_few_rows(t):
    """In the last elements of rows that end within a step, where a piece is read twice."""
    torch, sidco = _torch(), _sidco()
    for dim in (9, 37, 203):
        x, w = torch.ones(2, dim, dtype=_dtype(t), device="cuda"), torch.zeros(40, dim, dtype=_dtype(t), device="cuda")
        w[3, dim - 1], w[5, dim - 5], w[7, dim - 1] = float("inf"), float("-inf"), float("-inf")
        loss, lse = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
        sidco.sidco_cross_entropy(x, w, torch.tensor([1, 5], device="cuda"), loss, lse)
        assert lse.tolist() == [math.inf, math.inf] and loss.tolist() == [math.inf, math.inf]
        sidco.sidco_cross_entropy(x, w[4:], torch.tensor([0, 1], device="cuda"), loss, lse)
        # 36 words, two of them impossible
        assert abs(float(lse[0]) - math.log(34)) < 1e-6 * math.log(34) and loss[1] == math.inf


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_many_pieces_and_rows(t):
    """The gradient's pieces of the vocabulary, and the forward pass's of the rows."""
    torch = _torch()
    n, dim, vocab = 17_000, 24, 18_000 if t == "bf16" else 9000
    x, w, words = _case(n, dim, vocab, t, padding=0.3)
    g = torch.rand(n, device="cuda")
    loss, lse, dx, dw = _run(x, w, words, g)
    r = ref.CrossEntropy(x, w, words, g)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")
    _near(dx, *r.x_grad(), "x_grad")
    _near(dw, *r.w_grad(w.dtype), "w_grad")


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_padding_is_not_looked_at(t):
    torch, sidco = _torch(), _sidco()
    n, dim, vocab = 90, 72, 500
    x, w, words = _case(n, dim, vocab, t, padding=0.4)
    out = (words < 0) | (words >= vocab)
    x = x.contiguous()
    x[out] = 0.5
    first = _run(x, w, words)
    y = x.clone()
    y[out, ::3], y[out, 1::3] = float("nan"), float("inf")
    if t == "f32":
        y[out, 2::3] = 3e38
    second = _run(y, w, words)
    assert torch.equal(first[0], second[0]) and bool((first[0][out] == 0).all())
    assert torch.equal(first[1][~out], second[1][~out])
    assert torch.equal(first[2], second[2]) and bool((first[2][out] == 0).all())
    assert torch.equal(first[3], second[3])
    # nothing but padding
    nothing = torch.full_like(words, -1)
    loss, lse, dx, dw = _run(x, w, nothing)
    assert not bool(loss.any()) and not bool(dx.any()) and not bool(dw.any()) and bool(torch.isfinite(lse).all())
    before = torch.randn(vocab, dim, device="cuda")
    assert torch.equal(_run(x, w, nothing, None, None, before.to(x.dtype))[3], before.to(x.dtype))


def test_infinite_logits():
    torch = _torch()
    for t in ("f16", "bf16"):
        x = torch.zeros(5, 64, dtype=_dtype(t), device="cuda")
        w = torch.zeros(300, 64, dtype=_dtype(t), device="cuda")
        x[:, 0] = torch.tensor([1.0, -1.0, 0.0, 1.0, 1.0])
        w[7, 0] = float("inf")
        x[3, 1], w[:, 1] = float("-inf"), 1.0   # -inf for all but word 7, for which it is inf - inf
        x[4, 2] = float("nan")
        loss, lse, *_ = _run(x, w, torch.tensor([3, 3, 3, 3, 3], device="cuda"))
        lse = lse.tolist()
        assert lse[0] == math.inf and abs(lse[1] - math.log(299)) < 1e-6 * math.log(299) and math.isnan(lse[2])
        assert math.isnan(lse[3]) and math.isnan(lse[4])
        y = torch.zeros(1, 64, dtype=_dtype(t), device="cuda")
        y[0, 1] = float("-inf")
        loss, lse, *_ = _run(y, w[10:], torch.tensor([1], device="cuda"))
        assert lse.tolist() == [-math.inf]


@pytest.mark.parametrize("size", [1e-18, 1e-6, 300.0, 1e12])
def test_fp32_of_other_magnitudes(size):
    """x and w between them as usual, one large and the other small, and one row of w far below the others."""
    torch = _torch()
    x, w, words = _case(70, 100, 400, "f32")
    w = w.clone()
    w[5] *= 2.0**-12
    x, w = x / size, w * size
    g = torch.rand(70, device="cuda") * 1e-9
    loss, lse, dx, dw = _run(x, w, words, g)
    r = ref.CrossEntropy(x, w, words, g)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")
    _near(dx, *r.x_grad(), "x_grad")
    _near(dw, *r.w_grad(torch.float32), "w_grad")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(2.0**-20, 2.0**9), (2.0**9, 2.0**-20), (2.0**-14, 1.0), (1.0, 2.0**-14)])
def test_pieces_of_different_magnitudes(t, low, high):
    """The vocabulary's pieces are scaled for themselves, x once."""
    torch = _torch()
    n, dim, vocab = 17_000, 24, 18_000 if t == "bf16" else 9000
    x, w, words = _case(n, dim, vocab, t, padding=0.3)
    w = w.clone()
    w[:vocab // 2] *= low
    w[vocab // 2:] *= high
    x = x / max(low, high)
    g = torch.rand(n, device="cuda")
    loss, lse, dx, dw = _run(x, w, words, g)
    r = ref.CrossEntropy(x, w, words, g)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")
    _near(dx, *r.x_grad(), "x_grad")
    _near(dw, *r.w_grad(w.dtype), "w_grad")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_rows_gradients_of_other_magnitudes(t, size):
    """Its power of two and those of x and w have a product that no float holds."""
    torch = _torch()
    x, w, words = _case(70, 64, 520, t)
    g = torch.rand(70, device="cuda") * size
    loss, lse, dx, dw = _run(x, w, words, g)
    r = ref.CrossEntropy(x, w, words, g)
    _near(dx, *r.x_grad(), "x_grad")
    _near(dw, *r.w_grad(w.dtype), "w_grad")


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("x_size,w_size", [(2.0**-8, 2.0**8), (2.0**7, 2.0**-10), (2.0**-8, 1.0), (1.0, 2.0**-9)])
def test_one_gradient_alone_at_other_magnitudes(t, x_size, w_size):
    torch, sidco = _torch(), _sidco()
    for n, dim, vocab in ((70, 64, 520), (130, 72, 1024)):
        x, w, words = _case(n, dim, vocab, t)
        x, w = x * x_size, w * w_size
        loss, lse, dx, dw = _run(x, w, words)
        r = ref.CrossEntropy(x, w, words, None)
        _near(lse, r.lse, r.lse_off, "lse")
        _near(dx, *r.x_grad(), "x_grad")
        _near(dw, *r.w_grad(w.dtype), "w_grad")
        a, b = torch.empty_like(dx), torch.empty_like(dw)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, x_grad=a)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, weight_grad=b)
        torch.cuda.synchronize()
        assert torch.equal(a, dx) and torch.equal(b, dw)


def test_one_gradient_alone_and_losses_alone():
    torch, sidco = _torch(), _sidco()
    for t in ("f32", "bf16"):
        x, w, words = _case(100, 128, 900, t)
        loss, lse, dx, dw = _run(x, w, words)
        a, b = torch.empty_like(dx), torch.empty_like(dw)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, x_grad=a)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, weight_grad=b)
        one, other = torch.empty_like(loss), torch.empty_like(lse)
        sidco.sidco_cross_entropy(x, w, words, one, None)
        sidco.sidco_cross_entropy(x, w, words, None, other)
        torch.cuda.synchronize()
        assert torch.equal(a, dx) and torch.equal(b, dw) and torch.equal(one, loss) and torch.equal(other, lse)


def test_results_lie_within_their_rows():
    torch, sidco = _torch(), _sidco()
    for t in ("f32", "f16"):
        n, dim, vocab = 67, 30, 130
        x, w, words = _case(n, dim, vocab, t)
        loss, lse, dx, dw = _run(x, w, words)
        wx, ww = torch.full((n + 2, dim + 5), 9.0, dtype=x.dtype, device="cuda"), torch.full((vocab + 2, dim + 5), 9.0, dtype=x.dtype, device="cuda")
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, wx[1:-1, 3:3 + dim], ww[1:-1, 3:3 + dim])
        torch.cuda.synchronize()
        assert torch.equal(wx[1:-1, 3:3 + dim], dx) and torch.equal(ww[1:-1, 3:3 + dim], dw)
        for whole in (wx, ww):
            whole[1:-1, 3:3 + dim] = 9.0
            assert bool((whole == 9.0).all())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_no_loss_gradient_is_ones(t):
    """To the last bit, where probabilities are small too."""
    torch = _torch()
    for n, dim, vocab in ((3, 40, 30_000), (130, 64, 5000)):
        x, w, words = _case(n, dim, vocab, t)
        _, _, dx, dw = _run(x, w, words)
        _, _, ox, ow = _run(x, w, words, torch.ones(n, device="cuda"))
        assert torch.equal(dx, ox) and torch.equal(dw, ow)


@pytest.mark.parametrize("n", [3, 40])
def test_far_words(n):
    """Offsets into weight and gradient that pass 32 bits in elements and in bytes."""
    torch = _torch()
    dim, vocab = 2048, 1_100_000
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda").normal_(std=dim**-0.5, generator=gen)
    words = torch.randint(vocab - 2000, vocab, (n,), device="cuda", generator=gen)
    words[0] = 0
    x = (torch.randn(n, dim, device="cuda", generator=gen) + 4 * w[words]).bfloat16()
    loss, lse, dx, dw = _run(x, w, words)
    r = ref.CrossEntropy(x, w, words)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")
    _near(dx, *r.x_grad(), "x_grad")
    for part in (slice(0, 1000), slice(vocab // 2, vocab // 2 + 1000), slice(vocab - 2000, vocab)):
        r.p, r.p_off, keep = r.p[:, part], r.p_off[:, part], (r.p, r.p_off)
        _near(dw[part], *r.w_grad(w.dtype), ("w_grad", part))
        r.p, r.p_off = keep


def test_gradient_against_differences():
    """Central differences of the loss, for steps of one coordinate of x or w."""
    torch, sidco = _torch(), _sidco()
    n, dim, vocab, h = 6, 5, 40, 2.0**-5
    x, w, words = _case(n, dim, vocab, "f32", padding=0.2)
    x, w = x.contiguous(), w.contiguous()
    g = torch.rand(n, device="cuda")
    dx, dw = _run(x, w, words, g)[2:]
    r = ref.CrossEntropy(x, w, words, g)

    def f(x, w):
        loss = torch.empty(n, device="cuda")
        sidco.sidco_cross_entropy(x, w, words, loss, None)
        return float((loss.double() * r.g).sum())

    noise = 2 * float((r.loss_off * r.g.abs()).sum()) / h
    for m, grad, other in ((x, dx, w), (w, dw, x)):
        # the third derivative of log sum exp along a line is a third central moment of slopes within `range`, at most range^3 / 10
        span = 2 * float(other.abs().max())
        slack = h * h / 6 * span**3 / 10 * float(r.g.sum()) + noise
        for i in range(0, m.numel(), 7):
            up, down = m.clone(), m.clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            step = float(up.view(-1)[i].double() - down.view(-1)[i].double())
            slope = (f(up, w) - f(down, w) if m is x else f(x, up) - f(x, down)) / step
            assert abs(slope - float(grad.view(-1)[i])) <= slack + 1e-5, (i, slope, float(grad.view(-1)[i]), slack)


def test_the_same_every_time_on_two_streams_at_once():
    torch = _torch()
    sidco = _sidco()
    cases = [_case(300, 200, 2500, "bf16", seed=1), _case(150, 90, 1700, "f32", seed=2)]
    want = [_run(*c) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    torch.cuda.synchronize()
    for i in range(4):
        for (x, w, words), s in zip(cases, streams):
            with torch.cuda.stream(s):
                loss, lse = torch.empty(len(x), device="cuda"), torch.empty(len(x), device="cuda")
                dx, dw = torch.empty_like(x), torch.empty_like(w)
                sidco.sidco_cross_entropy(x, w, words, loss, lse)
                sidco.sidco_cross_entropy_grad(x, w, words, lse, None, dx, dw)
                outs.append((loss, lse, dx, dw))
    torch.cuda.synchronize()
    for k, o in enumerate(outs):
        assert all(torch.equal(a, b) for a, b in zip(o, want[k % 2]))
    for s in streams:
        sidco.sidco_release(stream=s)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_captured_and_replayed_beside_eager_calls(t):
    torch, sidco = _torch(), _sidco()
    n, dim, vocab = 140, 128, 1100
    x, w, words = _case(n, dim, vocab, t)
    x, w, words = x.contiguous(), w.contiguous(), words.clone()
    code = {"f32": sidco.GRAD_F32, "f16": sidco.GRAD_F16, "bf16": sidco.GRAD_BF16}[t]
    s = torch.cuda.Stream()
    loss, lse, dx, dw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    torch.cuda.synchronize()
    sidco.sidco_reserve(max(sidco.sidco_workspace_bytes_cross_entropy(n, dim, vocab, code),
                            sidco.sidco_workspace_bytes_cross_entropy_grad(n, dim, vocab, code, code)), stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        sidco.sidco_cross_entropy(x, w, words, loss, lse, stream=s)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, dx, dw, stream=s)
    for i in range(3):
        a, b, c = _case(n, dim, vocab, t, seed=10 + i, padding=0.2 * i)
        x.copy_(a * 2.0**i), w.copy_(b), words.copy_(c)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((loss, lse, dx, dw), _run(x, w, words)):
            assert torch.equal(got, want)
    del graph
    sidco.sidco_release(stream=s)


def test_reserved_memory_is_enough():
    torch, sidco = _torch(), _sidco()
    s = torch.cuda.Stream()
    for n, dim, vocab, t, gap in ((100, 96, 3000, "f32", 0), (100, 96, 3000, "bf16", 3), (700, 64, 500, "f16", 0)):
        x, w, words = _case(n, dim, vocab, t, gap=gap)
        code = {"f32": sidco.GRAD_F32, "f16": sidco.GRAD_F16, "bf16": sidco.GRAD_BF16}[t]
        loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        dx, dw = torch.empty(n, dim, dtype=x.dtype, device="cuda"), torch.empty(vocab, dim, device="cuda")
        need = max(sidco.sidco_workspace_bytes_cross_entropy(n, dim, vocab, code), sidco.sidco_workspace_bytes_cross_entropy_grad(n, dim, vocab, code, 0))
        space = torch.empty(need, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        sidco.sidco_set_workspace(space)  # of exactly this size: a call that needs more is refused
        try:
            sidco.sidco_cross_entropy(x, w, words, loss, lse, stream=s)
            sidco.sidco_cross_entropy_grad(x, w, words, lse, None, dx, dw, stream=s)
            sidco.sidco_cross_entropy_grad(x, w, words, lse, None, dx, stream=s)
            sidco.sidco_cross_entropy_grad(x, w, words, lse, None, None, dw, stream=s)
            torch.cuda.synchronize()
        finally:
            sidco.sidco_set_workspace(None)
