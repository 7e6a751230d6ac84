"""The layer operators' oracle against hand-worked and closed-form cases."""
import math

import numpy as np

import oracle
from oracle import layer


def test_bf16_rounding_is_nearest_even():
    one = 2.0 ** -7                                                 # bf16's step at 1
    x = np.array([1 + one / 2, 1 + 3 * one / 2, 1 + one / 4, -(1 + one / 2 + one / 64), 0.0, -0.0, 1e-40], np.float32)
    want = np.array([1.0, 1 + 2 * one, 1.0, -(1 + one), 0.0, -0.0, layer.round_bf16(np.float32([1e-40]))[0]], np.float32)
    assert np.array_equal(layer.round_bf16(x), want) and np.signbit(layer.round_bf16(x))[5]


def test_norm_by_hand():
    # z = (3, -4): mean square 12.5; weight (2, 1): v = (6, -4); d = 6 / 127; codes 127 and round(-84.67) = -85
    z, codes, delta = layer.rms_norm_quantize(np.float32([[1, -1]]), np.float32([2, 1]), 1e-6, "int8", residual=np.float32([[2, -3]]))
    assert z.tolist() == [[3, -4]]
    assert codes.view(np.int8).tolist() == [[127, -85]]
    assert abs(delta[0] - 6 / 127 / math.sqrt(12.5 + 1e-6)) < 1e-9


def test_norm_codes_are_those_of_the_normalised_row():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 64)).astype(np.float32)
    w = (1 + 0.1 * rng.standard_normal(64)).astype(np.float32)
    for fmt in ("int8", "e4m3", "e5m2"):
        _, codes, delta = layer.rms_norm_quantize(x, w, 1e-6, fmt)
        y = x.astype(np.float64) * w / np.sqrt((x.astype(np.float64) ** 2).mean(1, keepdims=True) + 1e-6)
        back = oracle.dequantize(codes, fmt, np.float32(delta))
        half_step = delta[:, None] * (0.5 if fmt == "int8" else np.maximum(np.abs(y / delta[:, None]) * 2.0 ** (-4 if fmt == "e4m3" else -3), 2.0 ** (-10 if fmt == "e4m3" else -17)))
        assert (np.abs(back - y) <= half_step * (1 + 1e-5)).all()


def test_norm_of_zeros():
    z, codes, delta = layer.rms_norm_quantize(np.zeros((2, 8), np.float32), np.ones(8, np.float32), 1e-6, "int8")
    assert not codes.any() and delta.tolist() == [1, 1]


def test_product_and_activations():
    cx = np.array([[1, -2, 3]], np.int8)
    cw = np.array([[4, 5, 6], [-7, 8, 9]], np.int8)
    assert layer.product_int8(cx, [0.5], cw, [2.0, 1.0]).tolist() == [[12.0, 2.0]]
    g = np.array([-30.0, -1.0, 0.0, 2.0, 500.0, -500.0])
    s = layer.activation(g, "silu")
    assert s[2] == 0 and s[4] == 500 and abs(s[3] - 2 / (1 + math.exp(-2))) < 1e-15 and abs(s[0] + 30 * math.exp(-30) / (1 + math.exp(-30))) < 1e-25
    e = layer.activation(g, "gelu")
    assert e[2] == 0 and e[4] == 500 and abs(e[1] + 0.15865525393145707) < 1e-15 and abs(e[3] - 2 * 0.9772498680518208) < 1e-14
    t = layer.activation(np.array([2.0, -1.0]), "gelu_tanh")
    for g1, t1 in ((2.0, t[0]), (-1.0, t[1])):
        assert abs(t1 - 0.5 * g1 * (1 + math.tanh(math.sqrt(2 / math.pi) * (g1 + 0.044715 * g1 ** 3)))) < 1e-14
