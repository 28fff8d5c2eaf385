"""Oracle for the paged cache in microscaled 4-bit floating point.  TEST INFRASTRUCTURE ONLY.

Format and page layout from their definition (block of 32 channels of a token; scale byte
s = max(e, 4) - 2 with e the bf16 exponent field of the largest magnitude; the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^(s - 127), ties to the even code, saturated; a block with an
infinity or a NaN: s = 255, codes 0), one value at a time, with numpy.
"""
from __future__ import annotations

import numpy as np

PAGE_BYTES = 2176
PAGE_TOKENS = 32
D = 128
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(bits):
    """bf16 bit patterns uint16 [n, 128] -> (codes uint8 [n, 128], scale bytes uint8 [n, 4])."""
    bits = np.asarray(bits, dtype=np.uint16)
    with np.errstate(invalid="ignore"):  # (signalling NaN)
        x = (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    n = bits.shape[0]
    codes, scales = np.zeros((n, D), np.uint8), np.zeros((n, 4), np.uint8)
    for t in range(n):
        for b in range(4):
            blk, u = x[t, 32 * b:32 * b + 32], bits[t, 32 * b:32 * b + 32]
            if not np.all(np.isfinite(blk)):
                scales[t, b] = 255
                continue
            s = max(int(((u & 0x7FFF) >> 7).max()), 4) - 2
            scales[t, b] = s
            y = np.abs(blk) / 2.0 ** (s - 127)
            d = np.abs(y[:, None] - GRID)
            near = d.min(axis=1, keepdims=True)
            for i in range(32):
                c = [j for j in range(8) if d[i, j] == near[i, 0]]
                c = c[0] if len(c) == 1 else [j for j in c if j % 2 == 0][0]
                codes[t, 32 * b + i] = c + (8 if u[i] >> 15 else 0)
    return codes, scales


def value(codes, scales):
    """codes [n, 128], scale bytes [n, 4] -> float64 [n, 128]."""
    c = np.asarray(codes).astype(int)
    s = np.repeat(np.asarray(scales).astype(float), 32, axis=-1)
    x = np.where(c >= 8, -1.0, 1.0) * GRID[c % 8] * 2.0 ** (s - 127)
    return np.where(s == 255, np.nan, x)


def places(values: bool):
    """For (token, channel) of a page: byte and nibble of the code; for (token, block): byte of the scale."""
    byte, nib = np.zeros((PAGE_TOKENS, D), int), np.zeros((PAGE_TOKENS, D), int)
    sc = np.zeros((PAGE_TOKENS, 4), int)
    for t in range(PAGE_TOKENS):
        q, j = t % 16 // 4, t % 4 + 4 * (t // 16)
        for c in range(D):
            if values:
                byte[t, c], nib[t, c] = 1024 * (c // 64) + 16 * (c % 16 + 16 * q) + 4 * (c // 16 % 4) + j // 2, j % 2
            else:
                byte[t, c], nib[t, c] = 64 * t + c // 2, c % 2
        for b in range(4):
            sc[t, b] = 2048 + (32 * q + 4 * j + b if values else 2 * (t % 16 + 16 * b) + t // 16)
    return byte, nib, sc


def put(page, t: int, codes, scales, values: bool) -> None:
    """Writes token t of a page (uint8 [2176], in place)."""
    byte, nib, sc = places(values)
    for c in range(D):
        a, sh = byte[t, c], 4 * nib[t, c]
        page[a] = (int(page[a]) & (0xF0 >> sh)) | (int(codes[c]) << sh)
    page[sc[t]] = scales


def get(page, values: bool):
    """A page's (codes [32, 128], scale bytes [32, 4])."""
    byte, nib, sc = places(values)
    return (page[byte] >> (4 * nib)) & 15, page[sc]


def page_values(page, values: bool):
    """A page's 32 tokens as float64 [32, 128]."""
    return value(*get(np.asarray(page), values))
