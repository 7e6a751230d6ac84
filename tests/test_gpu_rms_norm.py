"""qm_rms_norm_quantize against the oracle: codes and residual bit for bit, scales within what fp32 sums of squares may be off."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                   # half a step of fp32, relative
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def delta_tolerance(cols):
    # a sum of positive terms is off by at most the depth of additions a term passes through: a lane's own share of the row
    # (cols / 64 terms at least 64 lanes wide) and the tree above it, below 32; half of it survives the square root.  Then one
    # rounding each for the mean, eps, the root, the reciprocal, Eq. 1's division and the product
    return (((cols + 63) // 64 + 32) / 2 + 6) * U


def make(rows, cols, dtype, seed, pad=0, spread=1.0, lead=0):
    """[rows, cols] of a wider buffer whose other elements are NaN: nothing may read them."""
    g = torch.Generator().manual_seed(seed)
    wide = torch.full((rows, cols + pad), float("nan"), dtype=DT[dtype])
    x = torch.randn(rows, cols, generator=g) * spread
    x[:, ::13] *= 12.0
    wide[:, lead:lead + cols] = x.to(DT[dtype])
    return wide.cuda()[:, lead:lead + cols]


def check(x, w, eps, fmt, residual, got, delta_rows=slice(None)):
    codes, delta, z = got
    rows, cols = x.shape
    r = residual.float().cpu().numpy() if residual is not None else None
    want_z, want_codes, want_delta = layer.rms_norm_quantize(x.float().cpu().numpy(), w.float().cpu().numpy(), eps, fmt, r,
                                                             bf16=x.dtype == torch.bfloat16)
    c = codes.cpu().numpy()
    assert c.shape == (1, rows, qm.qm_code_ld(cols)) and not c[0, :, cols:].any()
    assert np.array_equal(c[0, :, :cols], want_codes)
    d = delta.cpu().numpy().astype(np.float64)
    assert (np.abs(d - want_delta) <= delta_tolerance(cols) * want_delta).all(), np.abs(d / want_delta - 1).max() / U
    if residual is None:
        assert z is None
    else:
        assert np.array_equal(z.float().cpu().numpy(), want_z)


SIZES = [(1, 1), (1, 2), (3, 7), (2, 8), (5, 15), (4, 16), (3, 17), (1, 64), (7, 100), (2, 128), (9, 255), (4, 256), (3, 257),
         (1, 768), (33, 1000), (2, 1024), (5, 1025), (3, 2048), (2, 2050), (301, 4096), (2, 4097), (3, 8192), (2, 8200),
         (2, 12288), (2, 16384), (1, 16400), (2, 30011), (1, 70001)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_against_oracle(rows, cols, dtype, fmt):
    x, r = make(rows, cols, dtype, 1), make(rows, cols, dtype, 2, spread=3.0)
    w = (1 + 0.1 * torch.randn(cols, generator=torch.Generator().manual_seed(3))).to(DT[dtype]).cuda()
    check(x, w, 1e-6, fmt, r, qm.qm_rms_norm_quantize(x, w, 1e-6, fmt, residual=r))
    check(x, w, 1e-5, fmt, None, qm.qm_rms_norm_quantize(x, w, 1e-5, fmt))


# more rows than SMs (several to a block), a length for each shape of the kernel, rows that start on 16 bytes and rows that do not
@pytest.mark.parametrize("rows,cols", [(1500, 200), (1700, 513), (5003, 700), (5000, 1001), (900, 1000), (900, 1001), (700, 1530), (701, 2041), (640, 3000), (650, 3001), (600, 4088),
                                       (610, 4095), (400, 6000), (400, 8185), (300, 12001), (200, 16384)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_more_rows_than_are_held_at_once(rows, cols, dtype, fmt):
    x, r = make(rows, cols, dtype, 20), make(rows, cols, dtype, 21, spread=3.0)
    w = (1 + 0.1 * torch.randn(cols, generator=torch.Generator().manual_seed(22))).to(DT[dtype]).cuda()
    check(x, w, 1e-6, fmt, r, qm.qm_rms_norm_quantize(x, w, 1e-6, fmt, residual=r))
    check(x, w, 1e-6, fmt, None, qm.qm_rms_norm_quantize(x, w, 1e-6, fmt))
    z = r.clone()                                                    # in place, every row ahead of its own writing
    check(x, w, 1e-6, fmt, r, qm.qm_rms_norm_quantize(x, w, 1e-6, fmt, residual=z, residual_out=z))


@pytest.mark.parametrize("rows,cols,pad,lead", [(5, 64, 8, 8), (5, 64, 8, 0), (4, 1024, 16, 16), (7, 1024, 3, 1), (3, 1000, 8, 8),
                                                (6, 999, 1, 1), (2, 4096, 64, 2), (3, 5000, 5, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("wdtype", ["bf16", "fp32"])
def test_pitches_and_offsets(rows, cols, pad, lead, dtype, wdtype):
    x, r = make(rows, cols, dtype, 4, pad, lead=lead), make(rows, cols, dtype, 5, pad + 8)
    w = torch.randn(cols + 1, generator=torch.Generator().manual_seed(6)).to(DT[wdtype]).cuda()[1:]      # off 16 bytes
    out = torch.full((rows, cols + pad), 7.0, dtype=DT[dtype], device="cuda")
    got = qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=r, residual_out=out[:, :cols])
    assert got[2].data_ptr() == out.data_ptr()
    check(x, w, 1e-6, "int8", r, got)
    assert (out[:, cols:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [100, 1024, 4096, 20000])
@pytest.mark.parametrize("which", ["x", "residual"])
def test_in_place(cols, which, dtype):
    x, r = make(6, cols, dtype, 7), make(6, cols, dtype, 8)
    w = torch.ones(cols, dtype=DT[dtype], device="cuda")
    x0, r0 = x.clone(), r.clone()
    got = qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=r, residual_out=x if which == "x" else r)
    check(x0, w, 1e-6, "int8", r0, got)
    assert torch.equal(*((r, r0) if which == "x" else (x, x0)))


@pytest.mark.parametrize("rows,cols", [(5, 101), (400, 1001), (300, 2048), (700, 4099), (4, 20001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_columns_beside_one_another(rows, cols, dtype):
    """x, the residual and its sum as columns of one buffer: the 16 bytes that two of them share are read beside their writing."""
    buf = torch.cat([make(rows, cols, dtype, 31), make(rows, cols, dtype, 32), make(rows, cols, dtype, 33)], 1)
    x, z, r = buf[:, :cols], buf[:, cols:2 * cols], buf[:, 2 * cols:]
    x0, r0 = x.clone(), r.clone()
    w = torch.ones(cols, device="cuda")
    check(x0, w, 1e-6, "int8", r0, qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=r, residual_out=z))
    assert torch.equal(x, x0) and torch.equal(r, r0)


def test_all_three_the_same_tensor():
    x = make(300, 1000, "bf16", 34)
    x0 = x.clone()
    w = torch.ones(1000, device="cuda")
    check(x0, w, 1e-6, "e4m3", x0, qm.qm_rms_norm_quantize(x, w, 1e-6, "e4m3", residual=x, residual_out=x))


@pytest.mark.parametrize("cols", [16, 1000, 1024, 4096, 20000])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_rows_that_are_zero_and_rows_that_are_not_finite(cols, fmt):
    x = make(8, cols, "bf16", 9)
    r = torch.zeros_like(x)
    w = torch.ones(cols, device="cuda")
    x[1] = 0.0
    x[2, cols // 2] = float("nan")
    x[3, 0] = float("inf")
    r[4, cols - 1] = float("-inf")
    r[5] = -x[5]                                                     # the sum is zero
    x[6, 3] = float("inf"); r[6, 3] = float("-inf")                   # the sum is NaN
    codes, delta, z = qm.qm_rms_norm_quantize(x, w, 1e-6, fmt, residual=r)
    d = delta.cpu()
    assert torch.isnan(d[[2, 3, 4, 6]]).all() and not codes[0, [1, 2, 3, 4, 5, 6]].any()
    assert d[1] == 1.0 and d[5] == 1.0
    rest = [0, 7]
    check(x[rest], w, 1e-6, fmt, r[rest], (codes[:, rest], delta[rest], z[rest]))
    assert torch.equal(z[:3].isnan(), (x + r)[:3].isnan())


def test_weights_that_leave_nothing_or_too_much():
    x = torch.ones(3, 64, device="cuda")
    x[1] = 1e20                                                      # squares beyond fp32
    x[2] = 2.0
    w = torch.zeros(64, device="cuda")
    codes, delta, _ = qm.qm_rms_norm_quantize(x, w, 1e-6, "e5m2")
    assert not codes.any() and delta[0] == 1.0 and torch.isnan(delta[1]) and delta[2] == 1.0
    w[5] = 3e38
    codes, delta, _ = qm.qm_rms_norm_quantize(x, w, 1e-6, "e5m2")
    assert torch.isfinite(delta[0]) and torch.isnan(delta[1]) and torch.isnan(delta[2])


def test_a_weight_that_is_not_finite_spoils_every_row():
    x = torch.ones(3, 100, device="cuda")
    x[1, 7] = 0.0
    for bad in (float("nan"), float("inf")):
        w = torch.ones(100, device="cuda")
        w[7] = bad
        codes, delta, _ = qm.qm_rms_norm_quantize(x, w, 1e-6, "int8")
        assert torch.isnan(delta).all() and not codes.any()


def test_residual_sums_of_any_bf16():
    """Any finite pair of bf16: the sum is the fp32 sum rounded to nearest even, subnormals, cancellation and overflow among it."""
    g = torch.Generator().manual_seed(30)
    bits = torch.randint(0, 1 << 16, (2, 512, 1024), generator=g, dtype=torch.int32)
    bits[1, 256:] = (bits[0, 256:] ^ 0x8000) + torch.randint(-2048, 2048, (256, 1024), generator=g, dtype=torch.int32)    # neighbours, mostly of the other sign
    bits &= 0xffff
    bits = torch.where((bits & 0x7f80) == 0x7f80, bits & 0x807f, bits)
    x, r = (b.to(torch.int16).view(torch.bfloat16) for b in bits)
    _, _, z = qm.qm_rms_norm_quantize(x.cuda(), torch.ones(1024, device="cuda"), 1e-6, "int8", residual=r.cuda())
    with np.errstate(over="ignore"):
        want = x.float().numpy() + r.float().numpy()
    finite = np.isfinite(want)
    got = z.float().cpu().numpy()
    assert np.array_equal(got[finite].view(np.uint32), layer.round_bf16(want[finite]).view(np.uint32))
    assert np.array_equal(got[~finite], want[~finite])


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e15])
def test_far_scales(scale):
    x = (torch.randn(4, 512, generator=torch.Generator().manual_seed(10)) * scale).cuda()
    w = torch.ones(512, device="cuda")
    check(x, w, 1e-6, "int8", None, qm.qm_rms_norm_quantize(x, w, 1e-6, "int8"))


@pytest.mark.parametrize("rows,cols", [(70000, 64), (200000, 16), (65537, 40), (100003, 1), (3001, 3)])
def test_many_short_rows(rows, cols):
    x = make(rows, cols, "bf16", 11)
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    check(x, w, 1e-6, "int8", x, qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=x))


def test_offsets_beyond_32_bits():
    rows, pitch = 3, (1 << 30) - 64                                 # elements: the last row starts beyond 2^32 bytes
    wide = torch.empty(2 * pitch + 1024, dtype=torch.bfloat16, device="cuda")
    x = wide.as_strided((rows, 1024), (pitch, 1))
    x.copy_(make(rows, 1024, "bf16", 12))
    w = torch.ones(1024, dtype=torch.bfloat16, device="cuda")
    check(x, w, 1e-6, "int8", None, qm.qm_rms_norm_quantize(x, w, 1e-6, "int8"))


def test_no_rows():
    w = torch.ones(64, device="cuda")
    codes, delta, z = qm.qm_rms_norm_quantize(torch.empty(0, 64, device="cuda"), w, 1e-6, "int8", residual=torch.empty(0, 64, device="cuda"))
    assert codes.shape == (1, 0, 64) and delta.shape == (0,) and z.shape == (0, 64)


def test_the_same_call_gives_the_same_bits():
    x = make(64, 4096, "bf16", 13)
    w = torch.ones(4096, device="cuda")
    a, b = (qm.qm_rms_norm_quantize(x, w, 1e-6, "e4m3", residual=x) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    c = qm.qm_rms_norm_quantize(x[7:8], w, 1e-6, "e4m3", residual=x[7:8])
    assert torch.equal(c[0][0, 0], a[0][0, 7])


def test_refusals():
    x, w = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for bad in (lambda: qm.qm_rms_norm_quantize(x.cpu(), w, 1e-6, "int8"), lambda: qm.qm_rms_norm_quantize(x, w.cpu(), 1e-6, "int8"),
                lambda: qm.qm_rms_norm_quantize(x.half(), w, 1e-6, "int8"), lambda: qm.qm_rms_norm_quantize(x, w.half(), 1e-6, "int8"),
                lambda: qm.qm_rms_norm_quantize(x.t(), torch.ones(4, device="cuda"), 1e-6, "int8"),
                lambda: qm.qm_rms_norm_quantize(x, w[:32], 1e-6, "int8"), lambda: qm.qm_rms_norm_quantize(x, w, 0.0, "int8"),
                lambda: qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=x[:3]),
                lambda: qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual=x.bfloat16()),
                lambda: qm.qm_rms_norm_quantize(x, w, 1e-6, "int8", residual_out=x),
                lambda: qm.qm_rms_norm_quantize(x[:1].expand(4, 64), w, 1e-6, "int8"),
                lambda: qm.qm_rms_norm_quantize(x[0], w, 1e-6, "int8"),
                lambda: qm.qm_rms_norm_quantize(x, w[:1].expand(64), 1e-6, "int8")):
        with pytest.raises(qm.QmError):
            bad()
