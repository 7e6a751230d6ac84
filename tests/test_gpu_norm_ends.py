"""qm_rms_norm_quantize at the ends of its range: long rows, rows next to nothing, large eps; and what its scales may be off."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                   # half a step of fp32, relative
# A term of a row of up to 16384 elements passes through at most 16 additions of its lane, one that joins the pair's halves, five of a warp
# and five of the block, half a step each; a longer row's lanes add with compensation, two half steps for any number of terms.  Half of
# that survives the square root; then one rounding each for the mean, eps, the root (which halves both), the reciprocal, Eq. 1's
# division and the product
REGISTERS, LONG = (27 / 2 + 6) * U, (12 / 2 + 6) * U


def expected(z, w, eps, qmax):
    """delta of float32 rows z in 64 bits."""
    v = (z * w[None, :]).astype(np.float32)
    return np.abs(v).max(1).astype(np.float64) / qmax / np.sqrt((z.astype(np.float64) ** 2).mean(1) + eps)


@pytest.mark.parametrize("cols", [1 << 20, (1 << 24) + 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
def test_scales_of_very_long_rows(cols, dtype, residual):
    """Equal elements, whose running sum in fp32 is off the same way at every addition."""
    value = 1.1
    x = torch.full((2, cols), value, device="cuda").to(dtype)
    x[1] *= -0.25
    w = torch.ones(cols, dtype=dtype, device="cuda")
    r = torch.zeros_like(x) if residual else None
    codes, delta, _ = qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=r)
    z = x.float().cpu().numpy()
    want = expected(z, np.ones(cols, np.float32), float(np.float32(1e-6)), 127)
    off = np.abs(delta.double().cpu().numpy() / want - 1)
    assert (off <= LONG).all(), off / U
    assert (codes[0, 0, :cols] == 127).all() and (codes[0, 1, :cols] == 129).all() and not codes[0, :, cols:].any()


@pytest.mark.parametrize("rows,cols", [(3, 100), (3, 1024), (600, 1024), (5, 2048), (400, 3000), (700, 4096), (300, 6000), (300, 8192), (200, 16384), (3, 16400), (2, 100001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
def test_scales_by_the_depth_of_their_sums(rows, cols, dtype, residual):
    g = torch.Generator(device="cuda").manual_seed(2)
    x, r = (torch.randn(rows, cols, device="cuda", generator=g).abs().to(dtype) for _ in range(2))
    w = (1 + 0.1 * torch.randn(cols, device="cuda", generator=g)).to(dtype)
    _, delta, z = qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=r if residual else None)
    want = expected((z if residual else x).float().cpu().numpy(), w.float().cpu().numpy(), float(np.float32(1e-6)), 127)
    off = np.abs(delta.double().cpu().numpy() / want - 1)
    assert (off <= (REGISTERS if cols <= 16384 else LONG)).all(), off.max() / U


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "e5m2"])
@pytest.mark.parametrize("cols", [40, 1000, 1024, 4096, 20001])
def test_rows_whose_scale_is_below_fp32(cols, fmt):
    """max|v| / qmax is 0 in fp32 although max|v| is not: the row counts as one of zeros, and its neighbours do not see it."""
    x = torch.randn(4, cols, generator=torch.Generator().manual_seed(1))
    x[1] = 0.0
    x[1, ::3] = 2.0 ** -149
    x[2, :] = -2.0 ** -148
    w = torch.ones(cols)
    codes, delta, _ = qm.qm_rms_norm_quantize(x.cuda(), w.cuda(), 1e-6, fmt)
    assert not codes[0, 1:3].any() and not codes[0, :, cols:].any()
    assert (delta[1:3] == 1.0).all()
    _, want, _ = layer.rms_norm_quantize(x[[0, 3]].numpy(), w.numpy(), 1e-6, fmt)
    assert np.array_equal(codes[0, [0, 3], :cols].cpu().numpy(), want)


@pytest.mark.parametrize("cols", [1, 8, 300, 20000])
@pytest.mark.parametrize("eps", [1.2e-38, 1e-20, 1e20, 3.4e38])
def test_scales_under_any_eps(cols, eps):
    """mean(z^2) + eps may leave fp32 where its root does not."""
    eps = float(np.float32(eps))
    x = torch.full((3, cols), 1.0)
    x[0] = 1.8e19 / cols ** 0.5 * 0.99                               # the sum of squares is near fp32's largest
    x[2] = 3e-3
    codes, delta, _ = qm.qm_rms_norm_quantize(x.cuda(), torch.ones(cols, device="cuda"), eps, "int8")
    want = expected(x.numpy(), np.ones(cols, np.float32), eps, 127)
    off = np.abs(delta.double().cpu().numpy() / want - 1)
    assert (off <= REGISTERS).all() and (codes[0, :, :cols] == 127).all()
