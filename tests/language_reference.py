"""A language model's operators in 64 bits, on the CPU and from their definitions: what the tests hold the kernels to."""
import numpy as np

M32 = 0xFFFFFFFF


def philox(counter, key):
    """Philox4x32-10 of one counter of four words and a key of two, in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def numbers(rows, cols, seed, offset):
    """The 16-bit numbers of rows x cols elements."""
    per_row = -(-cols // 8)
    block = np.arange(rows * per_row, dtype=np.uint64) + np.uint64(offset % 2**64)
    low, s32 = np.uint64(M32), np.uint64(32)
    c = [block & low, block >> s32, np.zeros_like(block), np.zeros_like(block)]
    k = [seed & M32, (seed >> 32) & M32]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> s32) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> s32) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    words = np.stack(c, -1)
    return np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(rows, per_row * 8)[:, :cols].astype(np.int64)


def dropout(x, p, seed, offset, residual=None):
    t = int(np.floor(65536 * p + 0.5))
    kept = numbers(*x.shape, seed, offset) >= t
    y = np.where(kept, x * (65536 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return y if residual is None else y + residual


def inside(words, vocab):
    return (words >= 0) & (words < vocab)


def embedding(table, words, scale):
    out = np.zeros((len(words), table.shape[1]))
    ok = inside(words, len(table))
    out[ok] = scale * table[words[ok]]
    return out


def embedding_grad(grad, words, vocab, scale):
    """The table's gradient, and beside it the same of the magnitudes and the number of rows of each word."""
    ok = inside(words, vocab)
    total, size = np.zeros((vocab, grad.shape[1])), np.zeros((vocab, grad.shape[1]))
    np.add.at(total, words[ok], grad[ok])
    np.add.at(size, words[ok], np.abs(grad[ok]))
    return scale * total, abs(scale) * size, np.bincount(words[ok], minlength=vocab)


class CrossEntropy:
    """Losses and gradients of x (n x k), w (v x k) in 64 bits, torch tensors wherever they lie, and how far from them results may
    be whose operands and sums are those that the calls document.

    u = 2^-24 is a rounding to 32 bits.  A logit is a sum of k products in 32 bits, off by at most (k + 16) u times the sum of
    their magnitudes; fp32 operands as pairs of halves miss 2^-22 of each factor and the product of what the first halves
    leave, 2^-22 again, and below the halves' range 2^-32 of the largest magnitude, which is 2^7 or more where a half is off
    by 2^-25 at least.  exp and log are those of powers of two, of an argument rounded to 32 bits twice.  P is rounded once to what it is stored in: a half for bf16 gradients, else a pair of
    halves, under a power of two of which its largest element may have 2^15; bf16 operands of its products are halves like
    fp32 ones, exactly but for that range."""

    def __init__(self, x, w, words, g=None):
        import torch
        f32 = x.dtype is torch.float32
        self.type, self.words, self.u = x.dtype, words.long(), 2.0**-24
        self.x, self.w = x.double(), w.double()
        self.ok = (self.words >= 0) & (self.words < len(w))
        self.x[~self.ok] = torch.where(torch.isfinite(self.x[~self.ok]), self.x[~self.ok], 0.0)
        k = x.shape[1]
        self.l = self.x @ self.w.t()
        size = self.x.abs() @ self.w.abs().t()
        self.l_off = ((k + 16) * self.u + (3 * 2.0**-22 if f32 else 0.0)) * size
        if f32:
            tops = self.x[self.ok].abs().max() if self.ok.any() else 0.0, self.w.abs().max()
            self.l_off += 2.0**-32 * (tops[0] * self.w.abs().sum(1)[None] + tops[1] * self.x.abs().sum(1)[:, None])
        self.lse = torch.logsumexp(self.l, 1)
        exponent = self.l_off + 4 * self.u * (self.l.abs() + self.lse.abs()[:, None])
        p = torch.exp(self.l - self.lse[:, None])
        # the exponentials' errors weighted by what they add, a sum in several steps, the result rounded
        self.lse_off = (p * torch.expm1(exponent)).sum(1) + 64 * self.u + 2 * self.u * self.lse.abs()
        at = torch.where(self.ok, self.words, 0)
        mine, mine_off = self.l.gather(1, at[:, None])[:, 0], exponent.gather(1, at[:, None])[:, 0]
        self.loss = torch.where(self.ok, self.lse - mine, 0.0)
        self.loss_off = torch.where(self.ok, self.lse_off + mine_off + 2 * self.u * self.loss.abs(), 0.0)
        g = torch.where(self.ok, torch.ones_like(self.lse) if g is None else g.double(), 0.0)
        self.p_off = g.abs()[:, None] * (p * torch.expm1(exponent + self.lse_off[:, None]) + 4 * self.u)
        p[torch.arange(len(x), device=x.device), at] -= 1
        self.p, self.g = p * g[:, None], g

    def _gradient(self, p, p_off, other, out):
        """p @ other, both in 64 bits, and the bound."""
        import torch
        f32 = self.type is torch.float32
        step = 2.0**-11 if out is torch.bfloat16 else 2.0**-22
        least = 2.0**-39 * float(self.g.abs().max())
        off = (p_off + p.abs() * step + least) @ other.abs()
        off = off + ((p.shape[1] + 16) * self.u + (3 * 2.0**-22 if f32 else 0.0)) * (p.abs() @ other.abs())
        if self.type is not torch.float16:
            off = off + 2.0**-32 * other.abs().max() * p.abs().sum(1)[:, None]
        info = torch.finfo(out)
        want = p @ other
        return want, off, info.eps / 2, info.tiny * info.eps / 2

    def x_grad(self):
        """(value, bound)"""
        want, off, rel, least = self._gradient(self.p, self.p_off, self.w, self.type)
        return want, off + (want.abs() + off) * rel + least

    def w_grad(self, out, before=None):
        import torch
        x = torch.where(self.ok[:, None], self.x, 0.0)
        want, off, rel, least = self._gradient(self.p.t(), self.p_off.t(), x, out)
        if before is not None:
            off = off + self.u * (before.double().abs() + want.abs())
            want = want + before.double()
        return want, off + (want.abs() + off) * rel + least
