"""The operators with a scale for each block, in float64 but for what their definition fixes in float32: FP8 codes under a scale for 128
contraction entries and their product; the 8-bit cache of keys and values and the attention that reads it.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
import numpy as np

from .formats import decode_table, qmax
from .probe import quantize

SIDE = 128


def quantize_blocks(x, fmt, side):
    """(codes [rows, K], delta [blocks of the contraction, blocks of rows]) of float32 x [rows, K]."""
    x = np.asarray(x, np.float32)
    rows, K = x.shape
    codes = np.zeros((rows, K), np.uint8)
    delta = np.ones((-(-K // SIDE), -(-rows // side)), np.float32)
    for c in range(delta.shape[0]):
        part = x[:, c * SIDE:(c + 1) * SIDE]
        with np.errstate(invalid="ignore"):
            top = np.array([np.abs(part[r:r + side]).max() for r in range(0, rows, side)], np.float32)
        good = np.isfinite(top)
        d = np.where(good, top, 0) / np.float32(qmax(fmt))                  # one float32 division
        delta[c] = np.where(good, np.where(d > 0, d, 1), np.nan).astype(np.float32)
        for r in range(delta.shape[1]):
            if good[r] and (d[r] > 0 or top[r] == 0):
                rs = slice(r * side, (r + 1) * side)
                codes[rs, c * SIDE:(c + 1) * SIDE] = quantize(part[rs], fmt, np.full(part[rs].shape[0], delta[c, r], np.float32))
    return codes, delta


def spread(delta, side, rows, K):
    """The scale of each element [rows, K]."""
    return np.repeat(np.repeat(np.asarray(delta, np.float64).T, side, 0)[:rows], SIDE, 1)[:, :K]


def product(cx, dx, fmt_x, cw, dw, fmt_w, side_w):
    """(y, the sum of its terms' magnitudes) [M, N]."""
    a = decode_table(fmt_x)[cx] * spread(dx, 1, *cx.shape)
    b = decode_table(fmt_w)[cw] * spread(dw, side_w, *cw.shape)
    return a @ b.T, np.abs(a) @ np.abs(b).T
