"""The dense operators in 64 bits, on the CPU and from their definitions: what the tests hold the kernels to."""
import numpy as np

SIZES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
MIDDLES = (SIZES[1:] + SIZES[:-1]) / 2


def mx4_blocks(x):
    """Rows of numbers -> (codes, exponent bytes) of their blocks, a code a byte, rows padded to 256."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    padded = -(-cols // 256) * 256
    b = np.zeros((rows, padded))
    b[:, :cols] = x
    b = b.reshape(rows, -1, 32)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(top)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.where(bad, 1.0, top)))
    # floor(log2) from the logarithm, mended where it was rounded across a power of two
    with np.errstate(over="ignore", invalid="ignore"):
        finite = (top > 0) & ~bad
        e = np.where(finite, e, -1000.0)
        e = np.where(finite & (np.exp2(e) > top), e - 1, e)
        e = np.where(finite & (np.exp2(e + 1) <= top), e + 1, e)
    byte = np.maximum(e - 2, -127) + 127
    small = np.abs(np.where(bad[..., None], 0.0, b)) / np.exp2(byte - 127)[..., None]
    low = np.searchsorted(MIDDLES, small, side="left")    # middles below it: a tie stays at the lower number
    high = np.searchsorted(MIDDLES, small, side="right")  # and goes up
    code = np.where(low % 2 == 0, low, high)              # to the even one of the two
    code = np.where(np.signbit(b) & ~bad[..., None], code + 8, code)
    return code.reshape(rows, padded).astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def mx4_pack(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def mx4_unpack(codes):
    out = np.empty((codes.shape[0], codes.shape[1] * 2), np.uint8)
    out[:, 0::2], out[:, 1::2] = codes & 15, codes >> 4
    return out


def mx4_values(code, byte, cols):
    """What codes (one a byte) and exponent bytes stand for."""
    v = SIZES[code & 7] * np.where(code & 8, -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (v.reshape(len(code), -1, 32) * scale[..., None]).reshape(len(code), -1)[:, :cols]


def rounded(x):
    """A matrix as the blocks of its rows stand for it."""
    return mx4_values(*mx4_blocks(x), np.asarray(x).shape[1])


def newton_schulz(x, steps, coef, eps):
    """X / (|X| + eps), then `steps` times X <- aX + (bA + cA^2)X with A = X X^T."""
    a, b, c = coef
    x = np.asarray(x, np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        if x.shape[0] > x.shape[1]:
            g = x.T @ x
            x = a * x + x @ (b * g + c * (g @ g))
        else:
            g = x @ x.T
            x = a * x + (b * g + c * (g @ g)) @ x
    return x
