"""The operators of a layer whose projections run in 8 bits, in float64 but for what their definition fixes in float32.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
import math

import numpy as np

from .formats import qmax
from .probe import quantize, scale


def round_bf16(x):
    """float64 or float32 values rounded to bf16 (nearest even), as float32."""
    w = np.ascontiguousarray(np.asarray(x, dtype=np.float32)).view(np.uint32).astype(np.uint64)
    w = (w + 0x7fff + ((w >> 16) & 1)) & 0xffff0000
    return w.astype(np.uint32).view(np.float32).reshape(np.shape(x))


def rms_norm_quantize(x, weight, eps, fmt, residual=None, bf16=False):
    """(z, codes, delta) of finite float32 arrays x, residual [rows, cols] and weight [cols]: z = x + residual in the
    stream's type (one float32 addition, then bf16 where the stream is that), v = z * weight in float32, codes of v under
    Eq. 1 per row, delta = Eq. 1's scale / rms(z) in float64 (1 where v is all zero)."""
    z = x if residual is None else (x + residual).astype(np.float32)
    if bf16 and residual is not None:
        z = round_bf16(z)
    v = (z * weight[None, :].astype(np.float32)).astype(np.float32)
    own = scale(v, fmt, "channel")
    codes = quantize(v, fmt, own)
    top = np.abs(v).max(axis=1).astype(np.float64)
    factor = 1.0 / np.sqrt((z.astype(np.float64) ** 2).mean(axis=1) + float(np.float32(eps)))
    delta = np.where(top == 0, 1.0, top / qmax(fmt) * factor)
    return z, codes, delta


def product_int8(cx, dx, cw, dw):
    """(sum_k x_ik w_jk) dx_i dw_j of int8 arrays [M, K], [N, K] and float32 scales."""
    acc = cx.astype(np.float64) @ cw.astype(np.float64).T          # exact: below 2^53
    return acc * (np.asarray(dx, np.float64)[:, None] * np.asarray(dw, np.float64)[None, :])


def activation(g, act):
    g = np.asarray(g, np.float64)
    if act == "silu":
        return g * _sigmoid(g)
    if act == "gelu":
        return 0.5 * g * np.array([math.erfc(-t / math.sqrt(2.0)) for t in g.ravel()]).reshape(g.shape)
    return g * _sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3))


def _sigmoid(t):
    e = np.exp(-np.abs(t))
    return np.where(t >= 0, 1.0, e) / (1.0 + e)
