"""qm_linear_int8 and qm_gated_linear_int8 against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                                   # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # of the output's type
TINY = 2.0 ** -125                                               # below this, products of scales leave fp32's normal range


def codes(rows, K, seed, pitch=None, full=False):
    """INT8 codes [rows, K], on the GPU as rows of `pitch` bytes whose rest is not zero: it must not be looked at."""
    g = torch.Generator().manual_seed(seed)
    c = torch.randint(-128 if full else -127, 128, (rows, K), generator=g, dtype=torch.int32).to(torch.int8)
    pitch = pitch or qm.qm_code_ld(K)
    wide = torch.randint(1, 128, (rows, pitch), generator=g, dtype=torch.int32).to(torch.int8)
    wide[:, :K] = c
    return c.numpy(), wide.view(torch.uint8).cuda()


def deltas(n, seed, scale):
    return (torch.rand(n, generator=torch.Generator().manual_seed(seed)) + 0.5) * scale


def within(y, want, tol, what):
    y = y.double().cpu().numpy()
    off = np.abs(y - want) - tol
    assert y.shape == want.shape and np.isfinite(y).all() and (off <= 0).all(), (what, off.max(), np.unravel_index(off.argmax(), off.shape))


def linear_tolerance(p, y, dt):
    # the int32 sum to fp32, the product of the scales, their product, the bias: a half step each, then the output's type
    return 3.01 * U * np.abs(p) + (1.01 * U + 1.01 * HALF[dt]) * np.abs(y) + TINY


def act_and_slope(g, act):
    """act(g) in 64 bits, |act'(g)| by differences, and how far an fp32 evaluation of act at an fp32 g may be off."""
    a = layer.activation(g, act)
    h = 1e-6 * np.maximum(1.0, np.abs(g))
    slope = np.abs(layer.activation(g + h, act) - layer.activation(g - h, act)) / (2 * h) * (1 + 1e-5) + 1e-9
    if act == "gelu":
        # 0.5 g (1 + erf(g / sqrt 2)): erf within 2 ulp of at most 1, the argument's rounding times erf's slope (at most
        # 0.42 g U / U), the sum's and the products' roundings; absolute, since 1 + erf cancels
        return a, slope, np.abs(g) * 6 * U + np.abs(a) * 3 * U
    # g / (1 + exp(t)) with t = -g, or the tanh form's t (five roundings): exp's argument is off by t's error, an error of
    # d there is d relative in exp, which is at most two ulp (4 U) off besides; sum and division a half step, division up to two ulp
    t = np.abs(g) if act == "silu" else 2 * np.sqrt(2 / np.pi) * np.abs(g + 0.044715 * g ** 3)
    return a, slope, np.abs(a) * ((2 if act == "silu" else 7) * np.minimum(t, 200.0) + 16) * U


def gated_reference(g, u, act, dt):
    a, slope, act_off = act_and_slope(g, act)
    h = a * u
    off = np.abs(u) * (slope * 3.01 * U * np.abs(g) + act_off) + np.abs(h) * (3.01 * U + 1.01 * U + 1.01 * HALF[dt])
    return h, 1.01 * off + TINY * (1 + np.abs(u))


SHAPES = [(1, 1, 1), (1, 64, 16), (1, 130, 17), (2, 3, 5), (3, 7, 128), (4, 256, 1024), (8, 129, 127), (9, 200, 129), (16, 128, 256),
          (17, 257, 100), (31, 64, 1000), (32, 1000, 512), (33, 384, 640), (64, 512, 2048), (65, 100, 300), (100, 1025, 96),
          (127, 128, 64), (128, 128, 128), (129, 255, 1008), (200, 640, 3000), (256, 256, 256), (257, 300, 333), (300, 2031, 1000),
          (512, 512, 512), (513, 1030, 130), (1, 4096, 4096), (5, 96, 8192), (770, 130, 64), (1000, 72, 1111), (2100, 520, 200),
          (4099, 1, 40), (1, 9001, 33)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_linear(M, N, K, dt):
    cx, x = codes(M, K, 1)
    cw, w = codes(N, K, 2)
    dx, dw = deltas(M, 3, 0.01), deltas(N, 4, 0.001)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(5))
    p = layer.product_int8(cx, dx.numpy(), cw, dw.numpy())
    y = qm.qm_linear_int8(x, dx.cuda(), w, dw.cuda(), K, out_dtype=dt)
    assert y.dtype == dt and tuple(y.shape) == (M, N)
    within(y, p, linear_tolerance(p, p, dt), "plain")
    for b in (bias, bias.bfloat16()):
        want = p + b.double().numpy()[None, :]
        within(qm.qm_linear_int8(x, dx.cuda(), w, dw.cuda(), K, bias=b.cuda(), out_dtype=dt), want, linear_tolerance(p, want, dt), "bias")


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gated(M, N, K, act):
    dt = torch.float32 if (M + N) % 2 else torch.bfloat16
    cx, x = codes(M, K, 6)
    cg, gate = codes(N, K, 7)
    cu, up = codes(N, K, 8)
    std = 127 * 127 / 3 * np.sqrt(K)                                # of the int32 sums
    dx, dg, du = deltas(M, 9, 0.01), deltas(N, 10, 300.0 / std), deltas(N, 11, 100.0 / std)     # g of a few units
    g = layer.product_int8(cx, dx.numpy(), cg, dg.numpy())
    u = layer.product_int8(cx, dx.numpy(), cu, du.numpy())
    h = qm.qm_gated_linear_int8(x, dx.cuda(), gate, dg.cuda(), up, du.cuda(), K, act=act, out_dtype=dt)
    assert h.dtype == dt and tuple(h.shape) == (M, N)
    want, tol = gated_reference(g, u, act, dt)
    within(h, want, tol, act)


# A shape for each way in which the products are cut on 148 SMs (rows of x per tile and parts of the contraction; then tiles of CTA pairs,
# several to a pair, in outputs whose rows start on 16, 8, 4 and 2 bytes)
CUTS = [(1, 4450, 907), (1, 65, 782), (1, 65, 1552), (17, 9483, 16), (18, 4509, 1708), (569, 129, 1435), (261, 129, 1801), (257, 135, 1400),
        (237, 65, 3597), (2475, 131, 16), (1240, 130, 2525), (593, 129, 2919), (559, 67, 5833), (265, 135, 6829), (67, 9615, 16),
        (2547, 135, 4553), (2251, 69, 5896), (2398, 135, 7447),
        (3333, 2600, 144), (3333, 2604, 144), (3333, 2603, 144), (6000, 2050, 1000), (6001, 2051, 1000), (411, 9936, 16)]


@pytest.mark.parametrize("M,N,K", CUTS)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_every_cut(M, N, K, dt):
    cx, x = codes(M, K, 50)
    cw, w = codes(N, K, 51)
    cu, up = codes(N, K, 52)
    std = 127 * 127 / 3 * np.sqrt(K)
    dx, dw, du = deltas(M, 53, 0.01), deltas(N, 54, 300.0 / std), deltas(N, 55, 100.0 / std)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(56))
    g = layer.product_int8(cx, dx.numpy(), cw, dw.numpy())
    u = layer.product_int8(cx, dx.numpy(), cu, du.numpy())
    want = g + bias.double().numpy()[None, :]
    within(qm.qm_linear_int8(x, dx.cuda(), w, dw.cuda(), K, bias=bias.cuda(), out_dtype=dt), want, linear_tolerance(g, want, dt), "linear")
    want, tol = gated_reference(g, u, "silu", dt)
    within(qm.qm_gated_linear_int8(x, dx.cuda(), w, dw.cuda(), up, du.cuda(), K, act="silu", out_dtype=dt), want, tol, "gated")


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M", [3, 300])
def test_gated_far_out(act, M):
    """Gates from -600 to 600: no NaN where exp leaves fp32's range."""
    N = 160
    one = torch.ones(M, 16, dtype=torch.int8)
    gate = torch.full((N, 16), 1, dtype=torch.int8)
    dg = torch.linspace(-600, 600, N) / 16
    g = layer.product_int8(one.numpy(), np.ones(M), gate.numpy(), dg.numpy())
    h = qm.qm_gated_linear_int8(one.view(torch.uint8).cuda(), torch.ones(M).cuda(), gate.view(torch.uint8).cuda(), dg.cuda(),
                                gate.view(torch.uint8).cuda(), torch.ones(N).cuda() / 16, 16, act=act, out_dtype=torch.float32)
    want, tol = gated_reference(g, np.ones_like(g), act, torch.float32)
    within(h, want, tol, act)


@pytest.mark.parametrize("M", [2, 40, 300, 600])
@pytest.mark.parametrize("K", [131071, 70000])
def test_longest_contraction(M, K):
    """Sums up to 2^31 - 2^14 in magnitude, codes of -128 among them."""
    cx, x = codes(M, K, 12, full=True)
    cw, w = codes(130, K, 13, full=True)
    x[0, :K] = 128; w[0, :K] = 128; w[1, :K] = 127                  # all -128: the largest sum; the other sign
    cx[0] = -128; cw[0] = -128; cw[1] = 127
    dx, dw = torch.ones(M), torch.ones(130)
    p = layer.product_int8(cx, dx.numpy(), cw, dw.numpy())
    assert p.max() == 128 * 128 * K
    within(qm.qm_linear_int8(x, dx.cuda(), w, dw.cuda(), K, out_dtype=torch.float32), p, linear_tolerance(p, p, torch.float32), "long")


@pytest.mark.parametrize("M,N,K", [(5, 100, 100), (64, 256, 512), (300, 260, 200), (700, 515, 144)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 1, 8, 61])
def test_pitches(M, N, K, dt, pad):
    """Rows of wider tensors on every side; what lies between the rows of the output stays."""
    cx, x = codes(M, K, 14, pitch=qm.qm_code_ld(K) + 48)
    cw, w = codes(2 * N, K, 15, pitch=qm.qm_code_ld(K) + 16)
    dx, dw = deltas(M, 16, 0.01), deltas(2 * N, 17, 0.0001)
    wide = torch.full((M, N + pad + 3), 5.0, dtype=dt, device="cuda")
    out = wide[:, 3:3 + N] if pad else wide[:, :N]
    y = qm.qm_linear_int8(x, dx.cuda(), w[N:], dw[N:].cuda(), K, out=out)
    assert y.data_ptr() == out.data_ptr()
    p = layer.product_int8(cx, dx.numpy(), cw[N:], dw[N:].numpy())
    within(y, p, linear_tolerance(p, p, dt), "linear")
    h = qm.qm_gated_linear_int8(x, dx.cuda(), w[:N], dw[:N].cuda(), w[N:], dw[N:].cuda(), K, act="silu", out=out)
    want, tol = gated_reference(layer.product_int8(cx, dx.numpy(), cw[:N], dw[:N].numpy()), p, "silu", dt)
    within(h, want, tol, "gated")
    first = 3 if pad else 0
    assert (wide[:, :first] == 5.0).all() and (wide[:, first + N:] == 5.0).all()


@pytest.mark.parametrize("M", [1, 3, 20, 100, 260, 600])
def test_rows_are_independent_of_the_batch(M):
    """The same row gives the same bits in any batch, and NaN scales stay in their row and column."""
    K, N = 520, 300
    _, x = codes(600, K, 18)
    _, w = codes(N, K, 19)
    dx, dw = deltas(600, 20, 0.01).cuda(), deltas(N, 21, 0.01).cuda()
    whole = qm.qm_linear_int8(x, dx, w, dw, K)
    assert torch.equal(qm.qm_linear_int8(x[:M], dx[:M], w, dw, K), whole[:M])
    both = qm.qm_gated_linear_int8(x, dx, w, dw, w, dw, K)
    assert torch.equal(qm.qm_gated_linear_int8(x[:M], dx[:M], w, dw, w, dw, K), both[:M])
    dx2, dw2 = dx[:M].clone(), dw.clone()
    dx2[M // 2] = float("nan"); dw2[7] = float("nan")
    for y, clean in ((qm.qm_linear_int8(x[:M], dx2, w, dw2, K), whole), (qm.qm_gated_linear_int8(x[:M], dx2, w, dw2, w, dw, K), both)):
        assert y[M // 2].isnan().all() and y[:, 7].isnan().all()
        keep = torch.ones_like(y, dtype=torch.bool)
        keep[M // 2] = False; keep[:, 7] = False
        assert torch.equal(y[keep], clean[:M][keep])


def test_offsets_beyond_32_bits():
    """An output of more than 2^32 bytes, and rows of codes that start beyond 2^31."""
    M, N, K = 35000, 66000, 16
    cx, x = codes(M, K, 22)
    cw, w = codes(N, K, 23)
    dx, dw = deltas(M, 24, 0.01), deltas(N, 25, 0.01)
    y = qm.qm_linear_int8(x, dx.cuda(), w, dw.cuda(), K)
    rows, cols = [0, 1, 32530, 34999], [0, 31, 65535, 65999]
    p = layer.product_int8(cx[rows], dx.numpy()[rows], cw[cols], dw.numpy()[cols])
    within(y[rows][:, cols], p, linear_tolerance(p, p, torch.bfloat16), "output")
    del y
    pitch = (1 << 30) - 16
    wide = torch.empty(4 * pitch + 64, dtype=torch.uint8, device="cuda")
    far = wide.as_strided((5, 48), (pitch, 1))
    c5, x5 = codes(5, 48, 26)
    c7, w7 = codes(7, 48, 27)
    far.copy_(x5)
    dx, dw = deltas(5, 28, 0.01), deltas(7, 29, 0.01)
    p = layer.product_int8(c5, dx.numpy(), c7, dw.numpy())
    within(qm.qm_linear_int8(far, dx.cuda(), w7, dw.cuda(), 48, out_dtype=torch.float32), p, linear_tolerance(p, p, torch.float32), "rows")
    within(qm.qm_linear_int8(w7, dw.cuda(), far, dx.cuda(), 48, out_dtype=torch.float32), p.T, linear_tolerance(p.T, p.T, torch.float32), "weights")


def test_many_rows_and_many_columns():
    for M, N in ((600000, 5), (3, 600000)):
        cx, x = codes(M, 32, 30)
        cw, w = codes(N, 32, 31)
        dx, dw = deltas(M, 32, 0.01), deltas(N, 33, 0.01)
        p = layer.product_int8(cx, dx.numpy(), cw, dw.numpy())
        within(qm.qm_linear_int8(x, dx.cuda(), w, dw.cuda(), 32), p, linear_tolerance(p, p, torch.bfloat16), (M, N))


def test_no_rows():
    _, w = codes(64, 32, 34)
    d = torch.ones(64, device="cuda")
    none, no_scales = torch.empty(0, 32, dtype=torch.uint8, device="cuda"), torch.empty(0, device="cuda")
    assert qm.qm_linear_int8(none, no_scales, w, d, 32).shape == (0, 64)
    assert qm.qm_gated_linear_int8(none, no_scales, w, d, w, d, 32).shape == (0, 64)


def test_refusals():
    _, x = codes(4, 64, 35)
    _, w = codes(32, 64, 36)
    dx, dw = torch.ones(4, device="cuda"), torch.ones(32, device="cuda")
    f, g = qm.qm_linear_int8, qm.qm_gated_linear_int8
    for bad in (lambda: f(x.cpu(), dx, w, dw, 64), lambda: f(x, dx.cpu(), w, dw, 64), lambda: f(x, dx[:3], w, dw, 64),
                lambda: f(x, dx, w, dw.double(), 64), lambda: f(x, dx, w, dw, 65), lambda: f(x.view(torch.int8), dx, w, dw, 64),
                lambda: f(x, dx, w, dw, 0), lambda: f(x[:, 1:], dx, w, dw, 48), lambda: f(x, dx, w[:, ::2], dw, 32),
                lambda: f(x, dx, w, dw, 64, bias=dw[:31]), lambda: f(x, dx, w, dw, 64, bias=dw.half()),
                lambda: f(x, dx, w, dw, 64, out_dtype=torch.float16), lambda: f(x, dx, w, dw, 64, out=torch.empty(4, 31, device="cuda")),
                lambda: f(x, dx, w, dw, 64, out=torch.empty(32, 4, device="cuda").t()), lambda: f(x[0], dx[:1], w, dw, 64),
                lambda: f(x, dx, w, dw, 64, out=torch.empty(4, 32)), lambda: f(torch.cat([x, x]).view(2, 4, 64), dx, w, dw, 64),
                lambda: g(x, dx, w, dw, w[:31], dw[:31], 64), lambda: g(x, dx, w, dw, w, dw[:31], 64), lambda: g(x, dx, w.cpu(), dw, w, dw, 64)):
        with pytest.raises(qm.QmError):
            bad()
    with pytest.raises(KeyError):
        g(x, dx, w, dw, w, dw, 64, act="relu")


@pytest.fixture
def starved_producer():
    L = qm.lib()
    L.qm_debug_set_wait_limit_ns(2_000_000)                            # 2 ms instead of 1 s
    yield L
    L.qm_debug_stop_producer_after(0xffffffff)
    L.qm_debug_set_wait_limit_ns(0)


# one row split over a cluster (long contractions: every part has several blocks); a few, unsplit (many weight rows); many, one tile
# and several to a CTA pair
@pytest.mark.parametrize("M,N,K", [(1, 256, 8192), (40, 256, 4096), (8, 30000, 256), (600, 300, 384), (2500, 2600, 256)])
@pytest.mark.parametrize("stop_after", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
def test_wait_runs_out_and_the_kernel_returns(starved_producer, M, N, K, stop_after, gated):
    """The loading warp stops on request (nothing is in flight that is never awaited): the waits run into their limit, the outputs
    that could not be computed are NaN, and the next call is right."""
    cx, x = codes(M, K, 37)
    cw, w = codes(N, K, 38)
    dx, dw = deltas(M, 39, 0.01).cuda(), deltas(N, 40, 0.0001).cuda()
    call = (lambda: qm.qm_gated_linear_int8(x, dx, w, dw, w, dw, K)) if gated else (lambda: qm.qm_linear_int8(x, dx, w, dw, K))
    want = call()
    assert not want.isnan().any()
    starved_producer.qm_debug_stop_producer_after(stop_after)
    y = call()
    torch.cuda.synchronize()
    bad = y.isnan()
    assert bad.any() and torch.equal(y[~bad], want[~bad])
    if stop_after == 0:
        assert bad.all()
    starved_producer.qm_debug_stop_producer_after(0xffffffff)
    assert torch.equal(call(), want)
