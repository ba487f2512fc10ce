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
