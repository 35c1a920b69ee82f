"""Plain implementations in 64 bits, on the CPU, of the rotation of rows to their
positions and of rows in 4 bits."""
import numpy as np
import torch

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDERS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])         # between them, as multiples of 2^e
RANGE = {torch.bfloat16: (-125, 125), torch.float16: (-23, 13)}


def rotated(x, position, freq, interleaved=False, factor=1.0):
    """Rows x [tokens, heads, dim] (float64) at their positions; freq are the
    32-bit numbers that the call gets."""
    angle = np.asarray(position, dtype=np.float64)[:, None, None] * np.asarray(freq, dtype=np.float64)
    c, s = factor * np.cos(angle), factor * np.sin(angle)
    r, y = len(freq), x.copy()
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if interleaved else (slice(0, r), slice(r, 2 * r))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def partners(x, freq, interleaved=False):
    """|x1| + |x2| of each element's pair, 0 where nothing is rotated."""
    r, y = len(freq), np.zeros_like(x)
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if interleaved else (slice(0, r), slice(r, 2 * r))
    y[..., a] = y[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y


def to_codes(x, dtype):
    """(codes, bytes E) of x [..., dim], and how near a border or a change of E
    some element of each 32 lies, relative to the largest."""
    lo, hi = RANGE[dtype]
    x = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(x).max(-1)
    odd = ~np.isfinite(top)
    top = np.where(odd, 1.0, top)
    x = np.where(odd[..., None], 0.0, x)
    m, k = np.frexp(top)                                            # top = m 2^k, 1/2 <= m < 1
    e = np.where(m <= 0.875, k - 3, k - 2)
    e = np.clip(np.where(top == 0, lo, e), lo, hi)
    size = np.abs(x) / np.exp2(e.astype(np.float64))[..., None]
    code = np.zeros(x.shape, dtype=np.int64)
    for i, b in enumerate(BORDERS):                                 # a tie goes to the even code
        code += size > b if i % 2 == 0 else size >= b
    near = np.abs(size[..., None] - BORDERS).min((-1, -2))
    near = np.minimum(near, np.abs(m - 0.875)) / 8
    code = np.where(x < 0, code + 8, code)
    scale = np.where(odd, 255, e + 127)
    return np.where(odd[..., None], 0, code).reshape(*x.shape[:-2], -1), scale, near


def packed(code):
    return (code[..., ::2] + 16 * code[..., 1::2]).astype(np.uint8)


def from_codes(codes, scale):
    """Values of packed codes [..., dim / 2] with bytes E [..., dim / 32]."""
    codes, scale = np.asarray(codes), np.asarray(scale).astype(np.int64)
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    unit = np.where(scale == 255, np.nan, np.exp2(scale - 127.0))
    return x * np.repeat(unit, 32, -1)
