"""Plain NumPy oracle of the microscaled 4-bit format: blocks of 32 four-bit codes and a power-of-two scale byte.

Written from the format's definition (include/aiq.h), in float64 and integers; shares no code with the CUDA library.
"""
import numpy as np

BLOCK = 32
ELEMENTS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def row_bytes(k):
    return -(-k // 128) * 64


def scale_row_bytes(k):
    return -(-k // 512) * 16


def quantize(x):
    """float rows [R][K] -> (codes uint8 [R][row_bytes], scales uint8 [R][scale_row_bytes])."""
    x = np.asarray(x)
    rows, k = x.shape
    codes = np.zeros((rows, 2 * row_bytes(k)), np.uint8)
    scales = np.zeros((rows, scale_row_bytes(k)), np.uint8)
    for r in range(rows):
        for b in range(-(-k // BLOCK)):
            v = x[r, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
            if not np.all(np.isfinite(v)):
                scales[r, b] = 255
                continue
            top = np.abs(v).max()
            # 2^e <= top < 2^(e + 1); the largest value is to lie in [4, 8) units, the smallest unit is 2^-127
            e = -127 if top == 0.0 else max(int(np.frexp(top)[1]) - 3, -127)
            scales[r, b] = e + 127
            a = np.abs(v) * 2.0 ** -e
            step = np.where(a < 2.0, 0.5, np.where(a < 4.0, 1.0, 2.0))
            q = np.minimum(np.rint(a / step) * step, 6.0)            # rint: halfway to even, and an even multiple is an even code
            codes[r, b * BLOCK:b * BLOCK + len(v)] = np.searchsorted(ELEMENTS, q) + 8 * np.signbit(v)
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8), scales


def dequantize(codes, scales, k):
    """float64 values [R][K]."""
    c = np.zeros((codes.shape[0], 2 * codes.shape[1]), np.int64)
    c[:, 0::2] = codes & 15
    c[:, 1::2] = codes >> 4
    c = c[:, :k]
    v = np.array(ELEMENTS)[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.repeat(scales.astype(np.int64), BLOCK, axis=1)[:, :k]
    return np.where(s == 255, np.nan, v * 2.0 ** (s - 127.0))


def product(x, w, bias=None):
    """float64 x [M][K] * w [N][K]^T + bias."""
    y = x.astype(np.float64) @ w.astype(np.float64).T
    return y if bias is None else y + bias.astype(np.float64)
