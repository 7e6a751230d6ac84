"""qm_linear_fp8 in every way that it is cut, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import blocks
from oracle.formats import decode_table
from test_gpu_linear_fp8 import codes, tolerance, within

pytestmark = pytest.mark.gpu

# On 148 SMs. Rows of x to a tile and parts of the contraction, or the CTA pairs' kernel; a scale for 128 weight rows, and where that is
# another one, a scale for each
CUTS = [(24, 512, 8192),       # (16, 8)
        (40, 1000, 4096),      # (16, 4)
        (32, 1024, 4096),      # (32, 8)
        (100, 1000, 4096),     # (32, 4)
        (300, 1000, 2000),     # (32, 1)
        (128, 512, 8192),      # (16, 4), (64, 8)
        (256, 1024, 4096),     # (64, 4)
        (64, 8192, 8192),      # (64, 2)
        (1000, 1024, 2048),    # (64, 1)
        (200, 500, 16384),     # (32, 4), (128, 8)
        (1000, 1024, 4096),    # (128, 2)
        (770, 2031, 1000),     # (128, 1)
        (2048, 2048, 2048),    # pairs, a tile each
        (2560, 4096, 1152),    # pairs, up to three tiles
        (2600, 4104, 1030)]    # pairs, ragged


def product(cx, dx, fmt_x, cw, dw, fmt_w, side):
    """blocks.product, its matrix products in float64 on the GPU."""
    a = torch.from_numpy(decode_table(fmt_x)[cx] * blocks.spread(dx, 1, *cx.shape)).cuda()
    b = torch.from_numpy(decode_table(fmt_w)[cw] * blocks.spread(dw, side, *cw.shape)).cuda()
    return (a @ b.t()).cpu().numpy(), (a.abs() @ b.abs().t()).cpu().numpy()


@pytest.mark.parametrize("M,N,K", CUTS)
@pytest.mark.parametrize("side", [128, 1])
def test_cuts(M, N, K, side):
    cx, dx, x, x_delta = codes(M, K, "e5m2", 1, 1, 0.01)
    cw, dw, w, w_delta = codes(N, K, "e4m3", 2, side, 0.001)
    p, top = product(cx, dx, "e5m2", cw, dw, "e4m3", side)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(5)) * float(np.abs(p).max())
    want = p + bias.double().numpy()[None, :]
    for dt in (torch.bfloat16, torch.float32):
        y = qm.qm_linear_fp8(x, x_delta, w, w_delta, K, "e5m2", "e4m3", side_w=side, out_dtype=dt)
        within(y, p, tolerance(p, top, K, dt), dt)
        assert torch.equal(qm.qm_linear_fp8(x, x_delta, w, w_delta, K, "e5m2", "e4m3", side_w=side, out_dtype=dt), y)
        y = qm.qm_linear_fp8(x, x_delta, w, w_delta, K, "e5m2", "e4m3", side_w=side, bias=bias.cuda(), out_dtype=dt)
        within(y, want, tolerance(want, top, K, dt, True), (dt, "bias"))


@pytest.mark.parametrize("M,N,K", [(64, 2048, 2048), (1000, 1024, 4096), (2600, 4104, 1030)])
@pytest.mark.parametrize("side", [128, 1])
def test_nan_scales_stay_in_their_rows_and_columns(M, N, K, side):
    _, _, x, dx = codes(M, K, "e4m3", 5, 1, 0.01)
    _, _, w, dw = codes(N, K, "e4m3", 6, side, 0.01)
    dx[-1, 1] = float("nan")
    j = 300 if side == 1 else 2
    dw[3, j] = float("nan")
    y = qm.qm_linear_fp8(x, dx, w, dw, K, side_w=side)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[1] = True
    bad[:, j * side:(j + 1) * side] = True
    assert torch.equal(y.isnan(), bad)


@pytest.mark.parametrize("M,N,K", [(64, 2000, 2048), (1000, 1024, 4096), (2600, 4104, 1030)])
def test_pitches_and_what_lies_between(M, N, K):
    cx, dx, x, x_delta = codes(M, K, "e4m3", 3, 1, 0.01, pitch=(K + 63) // 16 * 16)
    cw, dw, w, w_delta = codes(N, K, "e4m3", 4, 128, 0.01, pitch=(K + 47) // 16 * 16)
    p, top = product(cx, dx, "e4m3", cw, dw, "e4m3", 128)
    for dt in (torch.bfloat16, torch.float32):
        for pitch, first in ((N + 7, 3), (N + 8, 8)):
            wide = torch.full((M + 2, pitch + 16), 77.0, dtype=dt, device="cuda")
            out = wide[1:M + 1, first:first + N]
            assert qm.qm_linear_fp8(x, x_delta, w, w_delta, K, out=out) is out
            within(out, p, tolerance(p, top, K, dt), (pitch, first))
            wide[1:M + 1, first:first + N] = 77.0
            assert (wide == 77.0).all()


def test_terms_of_one_sign():
    """No cancellation: what truncation takes away shows in full, in the CTA pairs' kernel and over a split contraction."""
    for M, N, K in ((2048, 2048, 2048), (64, 2048, 4096)):
        cx, dx, x, x_delta = codes(M, K, "e4m3", 1, 1, 0.01)
        cw, dw, w, w_delta = codes(N, K, "e4m3", 2, 128, 0.001)
        for c, t in ((cx, x), (cw, w)):
            c &= 0x7F
            t[:, :K] &= 0x7F
        p, top = product(cx, dx, "e4m3", cw, dw, "e4m3", 128)
        y = qm.qm_linear_fp8(x, x_delta, w, w_delta, K, out_dtype=torch.float32)
        within(y, p, tolerance(p, top, K, torch.float32), (M, N, K))
