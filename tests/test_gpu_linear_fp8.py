"""qm_quantize_blocks and qm_linear_fp8 against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import blocks
from oracle.formats import decode_table, positive_grid

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                                   # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # of the output's type
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def matrix(rows, K, seed, dtype, strided, spread=0.0):
    """x [rows, K] in either order in memory, pitches of a multiple of 8, what lies between the rows large; and its fp32 values."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g) * torch.exp(spread * torch.randn(rows, K, generator=g))
    x = x.to(dtype)
    outer, inner = (K, rows) if strided else (rows, K)
    wide = torch.full((outer, (inner + 7) // 8 * 8 + 8), 1e4).to(dtype)
    wide[:, :inner] = x.t() if strided else x
    view = wide.cuda()[:, :inner]
    return (view.t() if strided else view), x.float().numpy()


CODES = [(1, 1), (1, 128), (2, 127), (3, 129), (31, 16), (32, 512), (33, 513), (64, 1000), (65, 130), (127, 640), (128, 128), (129, 257), (200, 2050),
         (257, 384), (1000, 72), (5, 8192)]


@pytest.mark.parametrize("rows,K", CODES)
@pytest.mark.parametrize("side", [1, 128])
@pytest.mark.parametrize("strided", [False, True])
def test_codes(rows, K, side, strided):
    for dtype, fmt in ((torch.bfloat16, "e4m3"), (torch.float32, "e5m2"), (torch.float32, "e4m3"), (torch.bfloat16, "e5m2")):
        x, values = matrix(rows, K, rows + K, dtype, strided, spread=2.0)
        codes, delta = qm.qm_quantize_blocks(qm.operand_of(x, -1), fmt, side=side)
        want_codes, want_delta = blocks.quantize_blocks(values, fmt, side)
        assert tuple(codes.shape) == (rows, qm.qm_code_ld(K)) and tuple(delta.shape) == want_delta.shape
        c = codes.cpu().numpy()
        assert np.array_equal(delta.cpu().numpy(), want_delta) and np.array_equal(c[:, :K], want_codes) and not c[:, K:].any(), (dtype, fmt)


@pytest.mark.parametrize("side", [1, 128])
@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_codes_of_special_blocks(side, strided, fmt):
    """Zeros of both signs, blocks at the ends of fp32, subnormal scales, NaN and Inf beside sound blocks."""
    x = torch.randn(300, 700, generator=torch.Generator().manual_seed(7))
    x[0:128, 0:128] = 0.0
    x[3, 5] = -0.0
    x[128:256, 128:256] *= 1e36
    x[128:256, 256:384] *= 1e-37
    x[0:128, 256:384] = torch.randn(128, 128) * 1e-42
    x[256:, 0:128] = 1e-45                                       # delta is 0 in fp32
    x[7, 400] = float("nan")
    x[200, 520] = float("inf")
    x[260, 699] = float("-inf")
    v = (x.t().contiguous() if strided else x).cuda()
    v = torch.nn.functional.pad(v, (0, -v.shape[1] % 8))[:, :v.shape[1]]
    codes, delta = qm.qm_quantize_blocks(qm.operand_of(v.t() if strided else v, -1), fmt, side=side)
    want_codes, want_delta = blocks.quantize_blocks(x.numpy(), fmt, side)
    assert np.array_equal(delta.cpu().numpy(), want_delta, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy()[:, :700], want_codes)
    assert np.isnan(want_delta).sum() == 3 and (want_delta == 1).sum() >= 2


def codes(rows, K, fmt, seed, side, scale, pitch=None):
    """FP8 codes [rows, K] of all finite values alike, on the GPU as rows of `pitch` bytes whose rest is NaN: it must not be looked at."""
    rng = np.random.default_rng(seed)
    n = len(positive_grid(fmt))
    c = (rng.integers(0, n, (rows, K)) | rng.integers(0, 2, (rows, K)) << 7).astype(np.uint8)
    pitch = pitch or qm.qm_code_ld(K)
    wide = np.full((rows, pitch), 0x7F, np.uint8)
    wide[:, :K] = c
    d = ((rng.random((-(-K // 128), -(-rows // side))) + 0.5) * scale).astype(np.float32)
    return c, d, torch.from_numpy(wide).cuda(), torch.from_numpy(d).cuda()


def tolerance(y, top, K, dt, bias=False):
    """top: the sum of the terms' magnitudes. A block's 128 exact products are added in fp32 with truncation, 32 at a time in an order of the
    hardware's: at most 2 U of the block's magnitudes for each of the 32 + 4 levels of sums; then the product of the scales (U), the
    multiply-add into the running sum (U each of a block), the bias, and the output's rounding."""
    return (2 * 36 + 2 + -(-K // 128)) * U * top + ((2 if bias else 1) * U + 1.01 * HALF[dt]) * np.abs(y) + 1e-37


def within(y, want, tol, what):
    y = y.double().cpu().numpy()
    off = np.abs(y - want) - tol
    assert y.shape == want.shape and np.isfinite(y).all() and (off <= 0).all(), (what, off.max(), np.unravel_index(off.argmax(), off.shape))


SHAPES = [(1, 1, 1), (1, 64, 16), (1, 130, 17), (2, 3, 5), (3, 7, 128), (4, 256, 1024), (8, 129, 127), (9, 200, 129), (16, 128, 256),
          (17, 257, 100), (31, 64, 1000), (32, 1000, 512), (33, 384, 640), (64, 512, 2048), (65, 100, 300), (100, 1025, 96),
          (127, 128, 64), (128, 128, 128), (129, 255, 1008), (200, 640, 3000), (256, 256, 256), (257, 300, 333), (300, 2031, 1000),
          (512, 512, 512), (513, 1030, 130), (1, 4096, 4096), (5, 96, 8192), (770, 130, 64), (1000, 72, 1111), (2100, 520, 200),
          (4099, 1, 40), (1, 9001, 33), (2600, 2600, 400), (3333, 2603, 144), (3333, 2602, 144), (400, 4000, 2000)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("side", [128, 1])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_product(M, N, K, side, dt):
    fx, fw = [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")][(M + N + K + side) % 4]
    cx, dx, x, x_delta = codes(M, K, fx, 1, 1, 0.01)
    cw, dw, w, w_delta = codes(N, K, fw, 2, side, 0.001)
    p, top = blocks.product(cx, dx, fx, cw, dw, fw, side)
    y = qm.qm_linear_fp8(x, x_delta, w, w_delta, K, fx, fw, side_w=side, out_dtype=dt)
    assert y.dtype == dt and tuple(y.shape) == (M, N)
    within(y, p, tolerance(p, top, K, dt), "plain")
    bias = torch.randn(N, generator=torch.Generator().manual_seed(5)) * float(np.abs(p).max())
    for b in (bias, bias.bfloat16()):
        want = p + b.double().numpy()[None, :]
        within(qm.qm_linear_fp8(x, x_delta, w, w_delta, K, fx, fw, side_w=side, bias=b.cuda(), out_dtype=dt), want,
               tolerance(want, top, K, dt, True), "bias")


@pytest.mark.parametrize("M,N,K", [(1, 64, 512), (40, 300, 1000), (300, 700, 1300), (2000, 512, 640)])
def test_terms_of_one_sign(M, N, K):
    """No cancellation: what truncation takes away shows in full."""
    cx, dx, x, x_delta = codes(M, K, "e4m3", 1, 1, 0.01)
    cw, dw, w, w_delta = codes(N, K, "e4m3", 2, 128, 0.001)
    cx &= 0x7F
    cw &= 0x7F
    x[:, :K] &= 0x7F
    w[:, :K] &= 0x7F
    p, top = blocks.product(cx, dx, "e4m3", cw, dw, "e4m3", 128)
    y = qm.qm_linear_fp8(x, x_delta, w, w_delta, K, out_dtype=torch.float32)
    within(y, p, tolerance(p, top, K, torch.float32), "one sign")


@pytest.mark.parametrize("M", [1, 20, 100, 400])
def test_pitches_and_what_lies_between(M):
    N, K = 333, 200
    cx, dx, x, x_delta = codes(M, K, "e4m3", 3, 1, 0.01, pitch=272)
    cw, dw, w, w_delta = codes(N, K, "e4m3", 4, 128, 0.01, pitch=224)
    p, top = blocks.product(cx, dx, "e4m3", cw, dw, "e4m3", 128)
    for dt in (torch.bfloat16, torch.float32):
        for pitch, first in ((N + 7, 0), (N + 7, 3), (344, 8), (336, 0)):
            wide = torch.full((M + 2, pitch + 16), 77.0, dtype=dt, device="cuda")
            out = wide[1:M + 1, first:first + N]
            assert qm.qm_linear_fp8(x, x_delta, w, w_delta, K, out=out) is out
            within(out, p, tolerance(p, top, K, dt), (pitch, first))
            wide[1:M + 1, first:first + N] = 77.0
            assert (wide == 77.0).all()


@pytest.mark.parametrize("M", [3, 70, 600])
@pytest.mark.parametrize("side", [1, 128])
def test_nan_scales_stay_in_their_rows_and_columns(M, side):
    N, K = 500, 400
    cx, dx, x, x_delta = codes(M, K, "e4m3", 5, 1, 0.01)
    cw, dw, w, w_delta = codes(N, K, "e4m3", 6, side, 0.01)
    x_delta[2, 1] = float("nan")
    j = 130 if side == 1 else 1
    w_delta[0, j] = float("nan")
    y = qm.qm_linear_fp8(x, x_delta, w, w_delta, K, side_w=side, out_dtype=torch.float32).cpu().numpy()
    bad = np.zeros((M, N), bool)
    bad[1] = True
    bad[:, j * side:(j + 1) * side] = True
    assert np.array_equal(np.isnan(y), bad)


def test_same_bits_every_time_and_on_another_stream():
    for M, N, K in ((1, 4096, 4096), (64, 1024, 8192), (700, 900, 1100)):
        _, _, x, dx = codes(M, K, "e4m3", 8, 1, 0.01)
        _, _, w, dw = codes(N, K, "e4m3", 9, 128, 0.01)
        first = qm.qm_linear_fp8(x, dx, w, dw, K)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        other = qm.qm_linear_fp8(x, dx, w, dw, K, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(first, other) and torch.equal(first, qm.qm_linear_fp8(x, dx, w, dw, K))


def test_training_products():
    """Forward, input gradient and weight gradient of y = x W^T from the codes of each orientation, against the products of what the codes stand for."""
    T, N, K = 700, 520, 392
    g = torch.Generator().manual_seed(11)
    x, W, dy = torch.randn(T, K, generator=g).cuda(), (torch.randn(N, K, generator=g) * 0.02).cuda(), (torch.randn(T, N, generator=g) * 1e-6).cuda()
    op = qm.operand_of

    def held(codes, delta, fmt, side, K):
        d = delta.double().t().repeat_interleave(side, 0)[:codes.shape[0]].repeat_interleave(128, 1)[:, :K]
        return codes.view(FLOAT8[fmt])[:, :K].double() * d
    for a, fa, b, fb, side, k in ((op(x, -1), "e4m3", op(W, -1), "e4m3", 128, K), (op(dy, -1), "e5m2", op(W, -2), "e4m3", 128, N),
                                  (op(dy, -2), "e5m2", op(x, -2), "e4m3", 1, T)):
        ca, da = qm.qm_quantize_blocks(a, fa)
        cb, db = qm.qm_quantize_blocks(b, fb, side=side)
        y = qm.qm_linear_fp8(ca, da, cb, db, k, fa, fb, side_w=side, out_dtype=torch.float32)
        u, v = held(ca, da, fa, 1, k), held(cb, db, fb, side, k)
        want, top = (u @ v.t()).cpu().numpy(), (u.abs() @ v.abs().t()).cpu().numpy()
        within(y, want, tolerance(want, top, k, torch.float32), (fa, fb, side))
    # a weight's scales are the same squares in both orientations
    assert torch.equal(qm.qm_quantize_blocks(op(W, -1), "e4m3", side=128)[1], qm.qm_quantize_blocks(op(W, -2), "e4m3", side=128)[1].t())


def test_captured_and_replayed():
    M, N, K = 48, 640, 1536
    x, _ = matrix(M, K, 1, torch.bfloat16, False)
    w, _ = matrix(N, K, 2, torch.bfloat16, False)
    cw, dw = qm.qm_quantize_blocks(qm.operand_of(w, -1), "e4m3", side=128)

    def step():
        c, d = qm.qm_quantize_blocks(qm.operand_of(x, -1), "e4m3")
        return qm.qm_linear_fp8(c, d, cw, dw, K)
    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = step()
    for k in range(3):
        x.mul_(1.0 + k)
        graph.replay()
        assert torch.equal(y, step())


@pytest.mark.parametrize("M,N,K,stop", [(8, 256, 2048, 1), (100, 1000, 4096, 3), (1000, 1024, 2048, 2)])
def test_wait_that_runs_out_leaves_nan(M, N, K, stop):
    _, _, x, dx = codes(M, K, "e4m3", 12, 1, 0.01)
    _, _, w, dw = codes(N, K, "e4m3", 13, 128, 0.01)
    sound = qm.qm_linear_fp8(x, dx, w, dw, K)
    try:
        qm.lib().qm_debug_set_wait_limit_ns(2_000_000)
        qm.lib().qm_debug_stop_producer_after(stop)
        y = qm.qm_linear_fp8(x, dx, w, dw, K)
        torch.cuda.synchronize()
        assert torch.isnan(y).any()
        assert torch.equal(y[~torch.isnan(y)], sound[~torch.isnan(y)])
    finally:
        qm.lib().qm_debug_stop_producer_after(0xffffffff)
        qm.lib().qm_debug_set_wait_limit_ns(0)
    assert torch.equal(qm.qm_linear_fp8(x, dx, w, dw, K), sound)
