"""GPU: gradients of rows that know their word, whose probability is one but for what the loss says, to the loss's own precision."""
import pytest

import language_reference as ref
from test_gpu_cross_entropy import _dtype, _sidco, _torch

pytestmark = pytest.mark.gpu


def _known(n, t, gap=0):
    """Rows whose word's logit is 4 to 18 above 119 others."""
    torch = _torch()
    dim, vocab = 128, 120
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = 0.01 * normal(vocab, dim + gap)
    w[:, :vocab].fill_diagonal_(1.0) if not gap else w[:, gap:gap + vocab].fill_diagonal_(1.0)
    words = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    x = 0.1 * normal(n, dim + gap)
    x[torch.arange(n, device="cuda"), gap + words] += torch.linspace(4.0, 18.0, n, device="cuda")
    words[n // 2] = -1
    return x.to(_dtype(t))[:, gap:], w.to(_dtype(t))[:, gap:], words


class Known(ref.CrossEntropy):
    """P is off by what the difference of two logits is, relative to itself, in the row's word too: z = sum over the other words of
    exp(l - l_t) is a sum of terms off by both logits' errors, loss = log(1 + z) and P = exp(-loss) - 1 by no more, each rounded."""

    def __init__(self, x, w, words, g):
        torch = _torch()
        super().__init__(x, w, words, g)
        exponent = self.l_off + 4 * self.u * (self.l.abs() + self.lse.abs()[:, None])
        at = torch.where(self.ok, self.words, 0)
        own = exponent.gather(1, at[:, None])[:, 0]
        p = torch.exp(self.l - self.lse[:, None])
        off = p * torch.expm1(exponent + self.lse_off[:, None])
        known = -torch.expm1(-self.loss)
        rows = torch.arange(len(x), device=x.device)
        p[rows, at] = -known
        off[rows, at] = known * (torch.expm1(exponent.max(1).values + own) + 70 * self.u)
        self.p, self.p_off = p * self.g[:, None], off * self.g.abs()[:, None]


@pytest.mark.parametrize("n,gap", [(3, 0), (40, 1), (100, 0), (300, 3)])
@pytest.mark.parametrize("t,o", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_rows_that_know_their_word(n, gap, t, o):
    torch, sidco = _torch(), _sidco()
    x, w, words = _known(n, t, gap)
    g = 0.5 + torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dx, dw = torch.full(x.shape, 3.0, dtype=x.dtype, device="cuda"), torch.full(w.shape, 3.0, dtype=_dtype(o), device="cuda")
    sidco.sidco_cross_entropy(x, w, words, loss, lse)
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, dx, dw, loss=loss)
    torch.cuda.synchronize()
    r = Known(x, w, words, g)
    for got, (want, off) in ((dx, r.x_grad()), (dw, r.w_grad(_dtype(o)))):
        miss = (got.double() - want).abs()
        assert bool((miss <= off).all()), (float(miss.max()), (miss > off).nonzero()[:4].tolist())
    # Of a row that knows its word best as of the others.  Each of the 128 elements is off by half the type's smallest step besides,
    # which for halves is 2^-25: sqrt(128) 2^-25 = 3.4e-7 beside a gradient of 1e-6.
    last, info = slice(n - 1, n), torch.finfo(x.dtype)
    want = r.x_grad()[0][last]
    assert float((dx[last].double() - want).norm()) <= 4e-3 * float(want.norm()) + 128**0.5 * info.tiny * info.eps / 2
    assert not bool(dx[n // 2].any())


class Sums(Known):
    """Without the losses a word of which a row knows more than a quarter has minus the sum of the row's others, off by what they are and a sum in
    32 bits; one of which it knows less is exp(l - lse) - 1.  Near a quarter it may be either."""

    def __init__(self, x, w, words, g):
        torch = _torch()
        super().__init__(x, w, words, g)
        base = ref.CrossEntropy(x, w, words, g)
        rows, at = torch.arange(len(x), device=x.device), torch.where(self.ok, self.words, 0)
        p, off = self.p[rows, at].abs(), self.p_off.clone()
        off[rows, at] = 0.0
        sums = off.sum(1) + 70 * self.u * p
        one = base.p_off[rows, at]
        known = torch.exp(-self.loss)
        off[rows, at] = torch.where(known > 0.26, sums, torch.where(known < 0.24, one, torch.maximum(sums, one)))
        self.p_off = off


@pytest.mark.parametrize("n,gap", [(3, 0), (40, 1), (100, 0), (300, 3)])
@pytest.mark.parametrize("t,o", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("low", [0, 30])
def test_without_the_losses(n, gap, t, o, low):
    torch, sidco = _torch(), _sidco()
    x, w, words = _known(n, t, gap)
    x = x * torch.rand(n, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n + 1)).round().clamp(min=0.125).to(x.dtype)
    gen = torch.Generator(device="cuda").manual_seed(n)
    g = (0.5 + torch.rand(n, device="cuda", generator=gen)) * torch.exp2(-low * torch.rand(n, device="cuda", generator=gen))
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dx, dw = torch.full(x.shape, 3.0, dtype=x.dtype, device="cuda"), torch.full(w.shape, 3.0, dtype=_dtype(o), device="cuda")
    sidco.sidco_cross_entropy(x, w, words, loss, lse)
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, dx, dw)
    torch.cuda.synchronize()
    r = Sums(x, w, words, g)
    for got, (want, off) in ((dx, r.x_grad()), (dw, r.w_grad(_dtype(o)))):
        off = off + 2.0**-38 * float(g.max()) * 128  # P by words is rounded under two powers of two where a row has one of its own
        miss = (got.double() - want).abs()
        assert bool((miss <= off).all()), (float(miss.max()), (miss > off).nonzero()[:4].tolist())
    a, b = torch.empty_like(dx), torch.empty_like(dw)
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, x_grad=a)
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, weight_grad=b)
    torch.cuda.synchronize()
    assert torch.equal(a, dx) and torch.equal(b, dw)


def test_no_number_stays_one_without_the_losses():
    torch, sidco = _torch(), _sidco()
    for n in (3, 130):
        x, w = torch.ones(n, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(300, 64, dtype=torch.bfloat16, device="cuda")
        w[7, 0] = float("inf")
        words = torch.full((n,), 7, device="cuda")
        x[1], words[1] = 0.0, -1
        lse, dx, dw = torch.full((n,), float("inf"), device="cuda"), torch.empty_like(x), torch.empty_like(w)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, dx, dw)
        torch.cuda.synchronize()
        # the padding row's P is zeros, and its x_grad P w: zero times infinity in the first column
        assert bool(torch.isnan(dx[0]).all()) and not bool(dx[1, 1:].any()) and bool(torch.isnan(dw[7]).all())


def test_one_gradient_alone_from_the_losses():
    torch, sidco = _torch(), _sidco()
    for t in ("f32", "bf16"):
        x, w, words = _known(100, t)
        loss, lse = torch.empty(100, device="cuda"), torch.empty(100, device="cuda")
        sidco.sidco_cross_entropy(x, w, words, loss, lse)
        dx, dw, a, b = torch.empty_like(x), torch.empty_like(w), torch.empty_like(x), torch.empty_like(w)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, dx, dw, loss=loss)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, x_grad=a, loss=loss)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, None, weight_grad=b, loss=loss)
        torch.cuda.synchronize()
        assert torch.equal(a, dx) and torch.equal(b, dw)


def test_infinite_losses():
    """A word that cannot be has P = -loss_grad."""
    torch, sidco = _torch(), _sidco()
    x, w = torch.ones(2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(300, 64, dtype=torch.bfloat16, device="cuda")
    x[1] = 0.0
    words = torch.tensor([5, 7], device="cuda")
    loss, lse = torch.tensor([float("inf"), 0.0], device="cuda"), torch.full((2,), 300.0, device="cuda").log()
    dw = torch.empty_like(w)
    sidco.sidco_cross_entropy_grad(x, w, words, lse, None, weight_grad=dw, loss=loss)
    torch.cuda.synchronize()
    want = torch.full((300,), 1 / 300)
    want[5] = -1.0
    # P in 11 bits, the gradient rounded to 8: half a step of each, and of lse 2^-21
    assert bool(((dw[:, 0].double().cpu() - want.double()).abs() <= want.double().abs() * (2.0**-12 + 2.0**-9 + 2.0**-20) * 1.01).all())
    assert torch.equal(dw, dw[:, :1].expand(300, 64))


def test_binding_refusals():
    torch, sidco = _torch(), _sidco()
    x, table = torch.zeros(6, 8, device="cuda"), torch.zeros(10, 8, device="cuda")
    words, lse, dx = torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(6, device="cuda"), torch.zeros(6, 8, device="cuda")
    for wrong, error in ((torch.zeros(5, device="cuda"), ValueError), (torch.zeros(6, dtype=torch.float64, device="cuda"), TypeError), (torch.zeros(6), TypeError)):
        with pytest.raises(error):
            sidco.sidco_cross_entropy_grad(x, table, words, lse, None, dx, loss=wrong)
