"""4-bit weights (MXFP4): 32 neighbours of a row share a scale 2^(s - 127); elements are 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
negatives.  Written element by element from the format's definition."""
import math

import numpy as np

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def nearest_code(a: float) -> int:
    """Code of the element nearest to the magnitude a, the even code halfway, 7 above."""
    best = min(range(8), key=lambda c: (abs(MAGNITUDES[c] - a), c % 2))
    return best


def quantize(W):
    """(codes [rows, cols / 2] uint8, scales [rows, cols / 32] uint8)."""
    W = np.asarray(W, dtype=np.float64)
    rows, cols = W.shape
    n = np.zeros((rows, cols), np.uint8)
    s = np.zeros((rows, cols // 32), np.uint8)
    for r in range(rows):
        for k in range(cols // 32):
            block = W[r, 32 * k:32 * k + 32]
            if not np.all(np.isfinite(block)):
                s[r, k] = 255
                continue
            top = float(np.max(np.abs(block)))
            e = -126 if top == 0 else max(-126, math.frexp(top)[1] - 1 - 2)
            s[r, k] = e + 127
            for i, w in enumerate(block):
                n[r, 32 * k + i] = nearest_code(math.ldexp(abs(float(w)), -e)) + (8 if np.signbit(w) else 0)
    return n[:, 0::2] | (n[:, 1::2] << 4), s


def dequantize(codes, scales):
    """The values, float64 (exact in bf16)."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    rows, half = codes.shape
    n = np.empty((rows, 2 * half), np.uint8)
    n[:, 0::2] = codes & 15
    n[:, 1::2] = codes >> 4
    table = np.array(MAGNITUDES + tuple(-m for m in MAGNITUDES))
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return table[n] * np.repeat(scale, 32, axis=1)
