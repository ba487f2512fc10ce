"""GPU: gradients of losses whose weights lie many powers of two apart: a row's x_grad is as near its own size as if it were alone."""
import pytest

import language_reference as ref
from test_gpu_cross_entropy import _case, _dtype, _run, _sidco, _torch

pytestmark = pytest.mark.gpu


class Rows(ref.CrossEntropy):
    """For x_grad a row's P has a power of two of its own from 2^8 below the largest on; for w_grad, where rows add up, one rounding under it
    and one under the common one, each of whose smallest step is 2^-39 of the largest or less."""

    def bound(self, p, p_off, other, out, least):
        """What _gradient says, with `least` for the smallest steps."""
        f32 = self.type is _dtype("f32")
        step = 2.0**-11 if out is _dtype("bf16") else 2.0**-22
        off = (p_off + p.abs() * step + least) @ other.abs()
        off = off + ((p.shape[1] + 16) * self.u + (3 * 2.0**-22 if f32 else 0.0)) * (p.abs() @ other.abs())
        if self.type is not _dtype("f16"):
            off = off + 2.0**-32 * other.abs().max() * p.abs().sum(1)[:, None]
        info = _torch().finfo(out)
        want = p @ other
        return want, off + (want.abs() + off) * info.eps / 2 + info.tiny * info.eps / 2

    def x_grad(self):
        own = self.g.abs()
        least = 2.0**-31 * own  # 2^-39 of the largest, which is less than 2^8 of the row's own
        return self.bound(self.p, self.p_off, self.w, self.type, least[:, None])

    def w_grad(self, out):
        x = _torch().where(self.ok[:, None], self.x, 0.0)
        return self.bound(self.p.t(), self.p_off.t(), x, out, 2.0**-38 * float(self.g.abs().max()))


def _weights(n, low, seed):
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    g = torch.rand(n, device="cuda", generator=gen) + 0.5
    return g * torch.exp2(-low * torch.rand(n, device="cuda", generator=gen)) * torch.where(torch.rand(n, device="cuda", generator=gen) < 0.5, -1.0, 1.0)


@pytest.mark.parametrize("n,dim,vocab", [(3, 40, 700), (70, 64, 520), (300, 130, 3000), (700, 256, 5000)])
@pytest.mark.parametrize("t,o", [("f32", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("low", [7, 20, 60])
def test_weights_far_apart(n, dim, vocab, t, o, low):
    torch = _torch()
    x, w, words = _case(n, dim, vocab, t)
    g = _weights(n, low, n) * (2.0**12 if t == "f16" else 1.0)
    g[0] = 2.0**12 if t == "f16" else 1.0
    g[n // 2] = 0.0
    _, _, dx, dw = _run(x, w, words, g, _dtype(o))
    r = Rows(x, w, words, g)
    for got, (want, off) in ((dx, r.x_grad()), (dw, r.w_grad(_dtype(o)))):
        miss = (got.double() - want).abs()
        assert bool((miss <= off).all()), (float((miss / off).max()), (miss > off).nonzero()[:4].tolist())


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_a_row_beside_a_much_larger_one(t):
    """As it is by itself, to the last bits."""
    torch = _torch()
    x, w, words = _case(2, 64, 30_000, t, padding=0.0)
    both = _run(x, w, words, torch.tensor([1.0, 2.0**-40], device="cuda"))[2]
    alone = _run(x[1:], w, words[1:], torch.tensor([2.0**-40], device="cuda"))[2]
    assert torch.equal(both[1:], alone) and bool(alone.any())


def test_pieces_and_splits():
    """A gradient of x that is put together from pieces of the vocabulary and of the contraction."""
    torch = _torch()
    for n, dim, vocab in ((17_000, 24, 9000), (40, 64, 60_000)):
        x, w, words = _case(n, dim, vocab, "f32", padding=0.3)
        g = _weights(n, 40, 5)
        _, _, dx, dw = _run(x, w, words, g)
        r = Rows(x, w, words, g)
        for got, (want, off) in ((dx, r.x_grad()), (dw, r.w_grad(torch.float32))):
            miss = (got.double() - want).abs()
            assert bool((miss <= off).all()), (float((miss / off).max()), (miss > off).nonzero()[:4].tolist())


def test_one_gradient_alone_and_weights_that_are_no_numbers():
    torch, sidco = _torch(), _sidco()
    for t in ("f32", "f16", "bf16"):
        x, w, words = _case(140, 72, 1100, t, padding=0.2)
        g = _weights(140, 30, 3)
        g[(words < 0) | (words >= 1100)] = float("nan")  # what stands in padding is not looked at
        _, lse, dx, dw = _run(x, w, words, g)
        a, b = torch.empty_like(dx), torch.empty_like(dw)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, g, x_grad=a)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, g, weight_grad=b)
        torch.cuda.synchronize()
        assert torch.equal(a, dx) and torch.equal(b, dw) and bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())
        g[5 if int(words[5]) in range(1100) else 6] = float("inf")
        _, _, dx, dw = _run(x, w, words, g)
        assert int((~torch.isfinite(dx)).any(1).sum()) <= 1
