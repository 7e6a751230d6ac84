"""Refusals of qm_rms_norm_quantize, qm_linear_int8 and qm_gated_linear_int8, on the host and without a GPU: every one is
found before anything is launched."""
import ctypes as C

import pytest

import paper_2408_02897_b200 as qm

INVALID, UNSUPPORTED, ALIGNMENT = 1, 2, 3
X, R, W, Z, CODES, DELTA = 0x100000, 0x200000, 0x300000, 0x400000, 0x500000, 0x600000


def norm(**over):
    a = dict(x=X, ld_x=64, residual=R, ld_residual=64, dtype=1, weight=W, weight_dtype=1, eps=1e-6, rows=8, cols=64, fmt=0,
             residual_out=Z, ld_out=64, codes=CODES, delta=DELTA, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_rms_norm_quantize(*a.values())


@pytest.mark.parametrize("over,status", [
    (dict(x=None), INVALID), (dict(weight=None), INVALID), (dict(codes=None), INVALID), (dict(delta=None), INVALID),
    (dict(residual=None), INVALID), (dict(residual_out=None), INVALID),              # both or neither
    (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(weight_dtype=7), INVALID), (dict(fmt=3), INVALID),
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=-5), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(eps=1e-39), INVALID),                                                       # not a normal fp32 number
    (dict(ld_x=63), INVALID), (dict(ld_residual=0), INVALID), (dict(ld_out=-64), INVALID),
    (dict(x=X + 1), ALIGNMENT), (dict(residual=R + 1), ALIGNMENT), (dict(residual_out=Z + 1), ALIGNMENT),
    (dict(weight=W + 1), ALIGNMENT), (dict(codes=CODES + 8), ALIGNMENT), (dict(delta=DELTA + 2), ALIGNMENT),
    (dict(dtype=0, x=X + 2), ALIGNMENT),
    (dict(residual_out=X + 2), INVALID), (dict(residual_out=R + 64), INVALID),         # overlaps in part
    (dict(residual_out=X, ld_out=128), INVALID),                                      # the same start, another pitch
    (dict(residual_out=X - 2, rows=1), INVALID),
    (dict(ld_x=128, ld_out=128, residual_out=X + 2 * 32), INVALID),                   # columns that overlap
    (dict(rows=1 << 31), UNSUPPORTED), (dict(cols=1 << 30, ld_x=1 << 30, ld_residual=1 << 30, ld_out=1 << 30), UNSUPPORTED),
    (dict(ld_x=1 << 30), UNSUPPORTED), (dict(ld_out=1 << 40), UNSUPPORTED),
])
def test_norm_refuses(over, status):
    assert norm(**over) == status


def test_norm_of_no_rows_does_nothing():
    assert norm(rows=0) == 0
    assert norm(rows=0, x=None, residual=None, weight=None, residual_out=None, codes=None, delta=None) == 0


def linear(**over):
    a = dict(codes_x=X, ld_x=64, delta_x=R, codes_w=W, ld_w=64, delta_w=Z, bias=CODES, bias_dtype=0, M=8, N=32, K=64,
             out=DELTA, out_dtype=1, ld_out=32, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_linear_int8(*a.values())


def gated(**over):
    a = dict(codes_x=X, ld_x=64, delta_x=R, codes_gate=W, ld_gate=64, delta_gate=Z, codes_up=W + 4096, ld_up=64, delta_up=Z + 512,
             act=0, M=8, N=32, K=64, out=DELTA, out_dtype=1, ld_out=32, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_gated_linear_int8(*a.values())


PRODUCT = [
    (dict(codes_x=None), INVALID), (dict(delta_x=None), INVALID), (dict(out=None), INVALID),
    (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(N=-3), INVALID),
    (dict(out_dtype=2), INVALID), (dict(ld_x=48), INVALID), (dict(ld_out=31), INVALID),
    (dict(codes_x=X + 8), ALIGNMENT), (dict(ld_x=72), ALIGNMENT), (dict(delta_x=R + 2), ALIGNMENT),
    (dict(out=DELTA + 1), ALIGNMENT), (dict(out_dtype=0, out=DELTA + 2), ALIGNMENT),
    (dict(M=1 << 31), UNSUPPORTED), (dict(N=1 << 30, ld_out=1 << 30), UNSUPPORTED), (dict(ld_x=1 << 30), UNSUPPORTED),
    (dict(ld_out=1 << 33), UNSUPPORTED),
]


@pytest.mark.parametrize("over,status", PRODUCT + [
    (dict(codes_w=None), INVALID), (dict(delta_w=None), INVALID), (dict(ld_w=63), INVALID), (dict(bias_dtype=5), INVALID),
    (dict(codes_w=W + 4), ALIGNMENT), (dict(ld_w=65), ALIGNMENT), (dict(delta_w=Z + 1), ALIGNMENT), (dict(bias=CODES + 2), ALIGNMENT),
    (dict(K=131072, ld_x=131072, ld_w=131072), UNSUPPORTED),
])
def test_linear_refuses(over, status):
    assert linear(**over) == status


@pytest.mark.parametrize("over,status", PRODUCT + [
    (dict(codes_gate=None), INVALID), (dict(codes_up=None), INVALID), (dict(delta_gate=None), INVALID), (dict(delta_up=None), INVALID),
    (dict(ld_gate=63), INVALID), (dict(ld_up=0), INVALID), (dict(act=3), INVALID), (dict(act=-1), INVALID),
    (dict(codes_up=W + 4), ALIGNMENT), (dict(ld_up=65), ALIGNMENT), (dict(delta_up=Z + 1), ALIGNMENT),
    (dict(K=131072, ld_x=131072, ld_gate=131072, ld_up=131072), UNSUPPORTED),
])
def test_gated_refuses(over, status):
    assert gated(**over) == status


def test_products_of_no_rows_do_nothing():
    assert linear(M=0) == 0 and gated(M=0) == 0
    assert linear(M=0, codes_x=None, delta_x=None, codes_w=None, delta_w=None, out=None) == 0


def test_missing_library_fails_loudly(monkeypatch):
    from paper_2408_02897_b200 import binding
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_LIB_PATH", "/nonexistent/libqm.so")
    with pytest.raises(qm.QmError):
        linear()
