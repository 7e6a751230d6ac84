"""Refusals of qm_quantize_blocks, qm_linear_fp8, qm_cache_append and qm_cache_attention, on the host and without a GPU: every one is found
before anything is launched."""
import ctypes as C

import pytest

import paper_2408_02897_b200 as qm
from paper_2408_02897_b200 import binding

INVALID, UNSUPPORTED, ALIGNMENT, SMALL = 1, 2, 3, 4
X, R, W, Z, CODES, DELTA, Q = 0x100000, 0x200000, 0x300000, 0x400000, 0x500000, 0x600000, 0x700000


def quantize(fmt=1, side=1, delta=DELTA, codes=CODES, **over):
    a = dict(data=X, dtype=1, noncontract=8, contract=64, stride_nc=64, stride_c=1, batch=1, stride_batch=0)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_quantize_blocks(C.byref(binding.Operand(*a.values())), fmt, side, delta, codes, None)


@pytest.mark.parametrize("over,status", [
    (dict(data=None), INVALID), (dict(delta=None), INVALID), (dict(codes=None), INVALID), (dict(dtype=2), INVALID), (dict(fmt=3), INVALID),
    (dict(fmt=0), UNSUPPORTED), (dict(side=2), INVALID), (dict(side=0), INVALID), (dict(side=64), INVALID), (dict(noncontract=0), INVALID),
    (dict(contract=-1), INVALID), (dict(batch=2, stride_batch=512), UNSUPPORTED), (dict(stride_nc=60), INVALID), (dict(stride_nc=68), ALIGNMENT),
    (dict(stride_c=2), UNSUPPORTED), (dict(data=X + 8), ALIGNMENT), (dict(codes=CODES + 8), ALIGNMENT), (dict(delta=DELTA + 2), ALIGNMENT),
    (dict(noncontract=1 << 31), UNSUPPORTED), (dict(contract=1 << 30, stride_nc=1 << 30), UNSUPPORTED),
    (dict(contract=1 << 24, stride_nc=1 << 24), UNSUPPORTED), (dict(side=128, noncontract=1 << 23), UNSUPPORTED),
])
def test_quantize_refuses(over, status):
    assert quantize(**over) == status


def linear(**over):
    a = dict(codes_x=X, ld_x=64, fmt_x=1, delta_x=R, codes_w=W, ld_w=64, fmt_w=2, delta_w=Z, side_w=128, bias=CODES, bias_dtype=0, M=8, N=32, K=64,
             out=DELTA, out_dtype=1, ld_out=32, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_linear_fp8(*a.values())


@pytest.mark.parametrize("over,status", [
    (dict(codes_x=None), INVALID), (dict(delta_x=None), INVALID), (dict(codes_w=None), INVALID), (dict(delta_w=None), INVALID), (dict(out=None), INVALID),
    (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(out_dtype=2), INVALID), (dict(bias_dtype=5), INVALID),
    (dict(fmt_x=3), INVALID), (dict(fmt_w=-1), INVALID), (dict(fmt_x=0), UNSUPPORTED), (dict(fmt_w=0), UNSUPPORTED), (dict(side_w=64), INVALID),
    (dict(ld_x=48), INVALID), (dict(ld_w=63), INVALID), (dict(ld_out=31), INVALID),
    (dict(codes_x=X + 8), ALIGNMENT), (dict(ld_x=72), ALIGNMENT), (dict(codes_w=W + 4), ALIGNMENT), (dict(ld_w=65), ALIGNMENT),
    (dict(delta_x=R + 2), ALIGNMENT), (dict(delta_w=Z + 1), ALIGNMENT), (dict(bias=CODES + 2), ALIGNMENT), (dict(out=DELTA + 1), ALIGNMENT),
    (dict(M=1 << 31), UNSUPPORTED), (dict(N=1 << 30, ld_out=1 << 30), UNSUPPORTED), (dict(ld_x=1 << 30), UNSUPPORTED),
    (dict(K=1 << 30, ld_x=1 << 30, ld_w=1 << 30), UNSUPPORTED),
])
def test_linear_refuses(over, status):
    assert linear(**over) == status


def test_product_of_no_rows_does_nothing():
    assert linear(M=0) == 0 and linear(M=0, codes_x=None, delta_x=None, codes_w=None, delta_w=None, out=None) == 0


CACHE = dict(k_codes=X, v_codes=R, k_delta=W, v_delta=W + 4096, blocks=8, kv_heads=2, block_tokens=16, head_dim=64, fmt=0, tables=Z, ld_tables=4,
             table_width=4, batch=3, lens=Z + 4096, starts=Z + 8192)


def cache_of(over):
    a = {k: over.pop(k, v) for k, v in CACHE.items()}
    return binding.Cache(*a.values())


def append(**over):
    c = cache_of(over)
    a = dict(k=CODES, ld_k=128, v=DELTA, ld_v=128, dtype=1, tokens=5, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_cache_append(C.byref(c), *a.values())


def attention(**over):
    c = cache_of(over)
    a = dict(q=CODES, ld_q=256, heads=4, scale=0.1, tokens=5, out=DELTA, ld_out=256, lse=Q, ws=0x10000000, ws_bytes=1 << 26, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return qm.lib().qm_cache_attention(C.byref(c), *a.values())


SHARED = [
    (dict(k_codes=None), INVALID), (dict(v_codes=None), INVALID), (dict(k_delta=None), INVALID), (dict(v_delta=None), INVALID),
    (dict(tables=None), INVALID), (dict(lens=None), INVALID), (dict(blocks=0), INVALID), (dict(kv_heads=0), INVALID), (dict(block_tokens=0), INVALID),
    (dict(head_dim=-16), INVALID), (dict(fmt=3), INVALID), (dict(table_width=0), INVALID), (dict(ld_tables=3), INVALID), (dict(batch=-1), INVALID),
    (dict(tokens=-1), INVALID), (dict(starts=None), INVALID),                           # then there are as many tokens as sequences
    (dict(block_tokens=8), UNSUPPORTED), (dict(block_tokens=48), UNSUPPORTED), (dict(block_tokens=512), UNSUPPORTED),
    (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=144), UNSUPPORTED), (dict(blocks=1 << 31), UNSUPPORTED),
    (dict(table_width=1 << 27, ld_tables=1 << 27), UNSUPPORTED), (dict(ld_tables=1 << 30), UNSUPPORTED),
    (dict(k_codes=X + 8), ALIGNMENT), (dict(v_codes=R + 1), ALIGNMENT), (dict(k_delta=W + 2), ALIGNMENT), (dict(tables=Z + 2), ALIGNMENT),
    (dict(lens=Z + 1), ALIGNMENT), (dict(starts=Z + 3), ALIGNMENT),
]


@pytest.mark.parametrize("over,status", SHARED + [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(dtype=2), INVALID), (dict(ld_k=120), INVALID), (dict(ld_v=0), INVALID),
    (dict(k=CODES + 8), ALIGNMENT), (dict(ld_k=132), ALIGNMENT), (dict(v=DELTA + 2), ALIGNMENT), (dict(ld_v=1 << 30), UNSUPPORTED),
])
def test_append_refuses(over, status):
    assert append(**over) == status


@pytest.mark.parametrize("over,status", SHARED + [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(ld_q=248), INVALID), (dict(ld_out=0), INVALID), (dict(ws=None), INVALID),
    (dict(q=CODES + 8), ALIGNMENT), (dict(ld_q=260), ALIGNMENT), (dict(out=DELTA + 2), ALIGNMENT), (dict(ws=0x10000010), ALIGNMENT), (dict(lse=Q + 2), ALIGNMENT),
    (dict(ws_bytes=100), SMALL), (dict(tokens=1 << 30, heads=4), UNSUPPORTED), (dict(ld_q=1 << 30), UNSUPPORTED),
])
def test_attention_refuses(over, status):
    assert attention(**over) == status


def test_nothing_to_do():
    none = dict(k_codes=None, v_codes=None, k_delta=None, v_delta=None, tables=None, lens=None)
    for empty in (dict(tokens=0), dict(batch=0, tokens=0, starts=None), dict(tokens=0, **none)):
        assert append(**empty) == 0 and attention(**empty) == 0
    assert attention(tokens=0, q=None, out=None, ws=None, ws_bytes=0) == 0 and append(tokens=0, k=None, v=None) == 0


def test_workspace():
    size = qm.lib().qm_cache_attention_workspace_bytes
    assert size(64) > 0 and size(128) > size(64) and size(80) == size(128) and size(0) == size(136) == size(256) == 0
