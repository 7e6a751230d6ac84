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


def cache_append(x, codes, delta, tables, lens, starts, fmt):
    """In place on codes [pages, heads, block, dim] (uint8) and delta [pages, heads] (float32): the new tokens x [tokens, heads, dim]."""
    block = codes.shape[2]
    table = decode_table(fmt).astype(np.float32)
    for b in range(len(lens)):
        first, end, length = int(starts[b]), int(starts[b + 1]), int(lens[b])
        for pos in range(max(0, length - (end - first)), length):
            if pos % block and pos != max(0, length - (end - first)):
                continue                                                     # not the first new one of its block
            page = tables[b][pos // block] if pos // block < tables.shape[1] else -1
            if not 0 <= page < codes.shape[0]:
                continue
            slot, n = pos % block, min(block - pos % block, length - pos)
            t0 = first + pos - (length - (end - first))
            for h in range(codes.shape[1]):
                new = np.asarray(x[t0:t0 + n, h], np.float32)
                with np.errstate(invalid="ignore"):
                    top = np.float32(np.abs(new).max())
                old = delta[page, h] if slot else np.float32(0)
                d = top / np.float32(qmax(fmt)) if np.isfinite(top) else np.float32(np.nan)
                d = np.float32(0) if d < 2.0 ** -60 else d
                d = old if old > d or np.isnan(old) else d
                if slot and d > old:
                    codes[page, h, :slot] = quantize(table[codes[page, h, :slot]] * old, fmt, np.full(slot, d, np.float32))
                codes[page, h, slot:slot + n] = quantize(new, fmt, np.full(n, d, np.float32)) if d > 0 else 0
                delta[page, h] = d


def cache_attention(q, kc, dk, vc, dv, tables, lens, starts, fmt, scale):
    """(out [tokens, heads, dim], lse [tokens, heads], and for tolerances the largest weighed magnitude of the values per output: sum p |v|)."""
    tokens, heads, dim = q.shape
    kv, block = kc.shape[1], kc.shape[2]
    table = decode_table(fmt)
    out, lse, top = np.zeros(q.shape), np.full((tokens, heads), -np.inf), np.zeros(q.shape)
    for b in range(len(lens)):
        first, end, length = int(starts[b]), int(starts[b + 1]), int(lens[b])
        if end <= first:
            continue
        n_blocks = -(-length // block)
        pages = [int(tables[b][i]) if i < tables.shape[1] else -1 for i in range(n_blocks)]
        good = [0 <= p < kc.shape[0] for p in pages]
        for h in range(heads):
            g = h // (heads // kv)
            def wide(codes, delta):
                parts = [table[codes[p, g]] * np.float64(delta[p, g] if not delta[p, g] < 2.0 ** -60 else 0) if ok else np.full((block, dim), np.nan)
                         for p, ok in zip(pages, good)]
                return np.concatenate(parts)[:length] if parts else np.zeros((0, dim))
            k, v = wide(kc, dk), wide(vc, dv)
            for t in range(first, end):
                seen = length - (end - 1 - t)
                if seen <= 0:
                    continue
                s = k[:seen] @ q[t, h].astype(np.float64) * scale
                m = s.max()
                p = np.exp(s - m)
                out[t, h] = p @ v[:seen] / p.sum()
                top[t, h] = p @ np.abs(v[:seen]) / p.sum()
                lse[t, h] = m + np.log(p.sum())
    return out, lse, top
