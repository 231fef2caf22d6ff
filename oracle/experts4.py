"""Expert matrices in 4 bits: what the library's format says, in numpy and fp64.

32 consecutive weights of a row (the inputs of one output) share 2^k, k the smallest integer with max|w| <= 6 2^k,
-127 <= k <= 125; a weight is the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} 2^k, a tie goes to the even code.
"""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK, CHUNK, TILE = 32, 128, 128


def weights4_encode(w):
    """w fp64 [..., C] -> codes 0..15 uint8 [..., C4], scale bytes uint8 [..., C4 / 32], C4 = C rounded up to 128."""
    w = np.asarray(w, dtype=np.float64)
    cols = w.shape[-1]
    pad = [(0, 0)] * (w.ndim - 1) + [(0, -cols % CHUNK)]
    blocks = np.pad(w, pad).reshape(*w.shape[:-1], -1, BLOCK)
    bad = ~np.isfinite(blocks).all(-1)
    blocks = np.where(bad[..., None], 0.0, blocks)
    top = np.abs(blocks).max(-1)
    k = np.full(top.shape, -127)
    for cand in range(-126, 126):                        # the smallest k that is large enough
        k = np.where(top > 6 * 2.0 ** (cand - 1), cand, k)
    a = np.abs(blocks) / (2.0 ** k)[..., None]
    off = np.abs(a[..., None] - VALUES)                  # distance to each value
    near = off.min(-1, keepdims=True)
    even_first = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = even_first[np.argmax((off == near)[..., even_first], -1)]
    code = code + 8 * np.signbit(blocks)
    code = np.where(bad[..., None], 0, code)
    scale = np.where(bad, 255, k + 127)
    return code.reshape(*w.shape[:-1], -1).astype(np.uint8), scale.astype(np.uint8)


def weights4_decode(code, scale, cols: int):
    """fp64 [..., cols]."""
    v = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    unit = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v.reshape(*scale.shape, BLOCK) * unit[..., None]).reshape(code.shape)[..., :cols]


def weights4_pack(code, scale):
    """[E, N, C4] codes and [E, N, C4 / 32] scale bytes -> the two arrays that the library takes."""
    E, N, blocks = scale.shape
    tiles, chunks = -(-N // TILE), blocks // 4
    out = np.zeros((E, tiles, chunks, 512), dtype=np.uint8)
    for n in range(N):
        for b in range(blocks):
            out[:, n // TILE, b // 4, n % 32 * 16 + n // 32 % 4 * 4 + b % 4] = scale[:, n, b]
    return code[..., 0::2] | code[..., 1::2] << 4, out
