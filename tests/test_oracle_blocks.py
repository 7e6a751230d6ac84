"""The oracle of the operators with a scale for each block, against loops and closed forms."""
import numpy as np
import pytest

from oracle import blocks
from oracle.formats import decode_table, qmax
from oracle.probe import quantize


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("side", [1, 128])
def test_blocks_are_quantized_one_by_one(fmt, side):
    x = np.random.default_rng(0).standard_normal((150, 300)).astype(np.float32) * np.exp(np.random.default_rng(1).standard_normal((150, 1)) * 3).astype(np.float32)
    codes, delta = blocks.quantize_blocks(x, fmt, side)
    assert delta.shape == (3, 150 if side == 1 else 2)
    for c in range(3):
        for r in range(delta.shape[1]):
            part = x[r * side:(r + 1) * side, c * 128:(c + 1) * 128]
            d = np.abs(part).max() / np.float32(qmax(fmt))
            assert delta[c, r] == d
            assert np.array_equal(codes[r * side:(r + 1) * side, c * 128:(c + 1) * 128], quantize(part, fmt, np.full(len(part), d, np.float32)))


def test_special_blocks():
    x = np.ones((130, 130), np.float32)
    x[:128, :128] = 0
    x[128, 0] = np.nan
    x[0, 129] = np.inf
    codes, delta = blocks.quantize_blocks(x, "e4m3", 128)
    assert delta[0, 0] == 1 and np.isnan(delta[0, 1]) and np.isnan(delta[1, 0]) and delta[1, 1] == np.float32(1) / np.float32(448)
    assert not codes[:128].any() and not codes[128:, :128].any() and (codes[128:, 128:] == 0x7E).all()


def test_product_is_the_sum_of_scaled_blocks():
    rng = np.random.default_rng(2)
    cx, cw = rng.integers(0, 0x70, (3, 200)).astype(np.uint8), rng.integers(0, 0x70, (130, 200)).astype(np.uint8)
    dx, dw = rng.random((2, 3)).astype(np.float32), rng.random((2, 2)).astype(np.float32)
    y, top = blocks.product(cx, dx, "e4m3", cw, dw, "e5m2", 128)
    a, b = decode_table("e4m3")[cx], decode_table("e5m2")[cw]
    for i in range(3):
        for j in (0, 127, 128, 129):
            want = sum(float(dx[c, i]) * float(dw[c, j // 128]) * (a[i, 128 * c:128 * c + 128] @ b[j, 128 * c:128 * c + 128]) for c in range(2))
            assert abs(y[i, j] - want) <= 1e-12 * abs(want) and top[i, j] == pytest.approx(want)


def test_append_grows_a_scale_and_starts_blocks_anew():
    codes, delta = np.full((2, 1, 16, 16), 0x55, np.uint8), np.full((2, 1), 7.0, np.float32)
    tables = np.array([[1, 0]])
    x = np.zeros((3, 1, 16), np.float32)
    x[0] = 1.27                                                   # alone: scale 0.01
    x[1], x[2] = 0.5, 2.54
    for n, want in ((1, 0.01), (2, 0.01), (3, 0.02)):
        blocks.cache_append(x[n - 1:n], codes, delta, tables, [n], [0, 1], "int8")
        assert delta[1, 0] == pytest.approx(want, rel=1e-6)
    assert (codes[1, 0, 0] == 64).all() and (codes[1, 0, 1] == 25).all() and (codes[1, 0, 2] == 127).all()     # 63.5 to even, 25
    assert (codes[1, 0, 3:] == 0x55).all() and (codes[0] == 0x55).all() and delta[0, 0] == 7


def test_attention_of_equal_keys_is_the_mean_of_what_is_seen():
    codes = np.zeros((2, 1, 16, 16), np.uint8)
    v = np.arange(32, dtype=np.uint8).reshape(2, 1, 16, 1).repeat(16, 3)
    one, q = np.ones((2, 1), np.float32), np.ones((3, 2, 16), np.float32)
    out, lse, top = blocks.cache_attention(q, codes, one, v, one, np.array([[0, 1]]), [20], [0, 3], "int8", 0.25)
    for t, seen in ((0, 18), (1, 19), (2, 20)):
        assert np.allclose(out[t], (seen - 1) / 2) and np.allclose(lse[t], np.log(seen)) and np.allclose(top[t], out[t])
