"""qm_cache_attention where the scales of a cache lie at the ends of their range, or far apart."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import blocks
from test_gpu_cache import U, Case, attention_tolerance, run_attention

pytestmark = pytest.mark.gpu

# (kv heads, group, head_dim, block, new tokens, lengths): rows of eight and 16, keys shared out among thread blocks, tiles
SHAPES = [(1, 4, 64, 16, [1, 1, 1], [700, 40, 129]), (2, 4, 128, 16, [3, 1, 9], [300, 5, 1000]), (16, 2, 64, 16, [130, 70], [190, 400]),
          (24, 4, 128, 32, [257, 64], [400, 90])]


def check(case, heads, **kw):
    q, out, lse, want, want_lse, top, scale = run_attention(case, heads, **kw)
    tol, tol_lse = attention_tolerance(case, q, want, top, scale)
    # there the exponent's roundings are of |x'| <= |x| log2 e + 80; log2 of a scale and the logarithm of a sum reach 140 here, and a term that is
    # taken again without its scale has two roundings more: 4 U (140 - 80) + 2 * 2 U 140 more of a weight, twice in a quotient
    more = 4 * U * 60 + 4 * U * 140
    tol, tol_lse = tol + 2 * more * (top + np.abs(want)), tol_lse + more
    assert np.isfinite(out).all()
    off = np.abs(out - want) - tol
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))
    off = np.abs(lse - want_lse) - tol_lse - 2 * U * np.abs(want_lse)
    assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("kv,group,dim,block,new,lens", SHAPES)
@pytest.mark.parametrize("least,most", [(126.0, 127.9), (120.0, 127.9), (-60.0, -58.0)])
def test_scales_of_values_at_the_ends(kv, group, dim, block, new, lens, least, most):
    """Codes of -1, 0 and 1 under scales up to fp32's largest: outputs that bf16 holds; and the least scales that count."""
    case = Case("int8", kv, dim, block, new, lens, seed=3).fill(lens)
    held = np.isfinite(case.dv)
    case.dv[held] = np.exp2(case.rng.uniform(least, most, case.dv.shape))[held].astype(np.float32)
    case.v[:] = np.where(case.v == 0x80, 0x80, (case.rng.integers(-1, 2, case.v.shape) & 0xFF)).astype(np.uint8)
    check(case, kv * group)


@pytest.mark.parametrize("kv,group,dim,block,new,lens", SHAPES)
@pytest.mark.parametrize("high", [90.0, 110.0, 127.0])
@pytest.mark.parametrize("order", ["mixed", "large ones first", "large ones last"])
def test_scales_of_values_far_apart(kv, group, dim, block, new, lens, high, order):
    """Blocks of nothing but zeros, and of scales of 2^-60 to 1, beside blocks of 2^high: their keys count in the denominator as any others."""
    case = Case("int8", kv, dim, block, new, lens, seed=5).fill(lens, scale_k=0.5)
    for b, n in enumerate(lens):
        pages = case.tables[b, :-(-n // block)]
        for h in range(kv):
            d = np.exp2(case.rng.choice([-61.0, -60.0, -40.0, 0.0, high], len(pages)) + case.rng.random(len(pages)) * 0.9)
            d[case.rng.random(len(pages)) < 0.2] = 0.0
            d = d if order == "mixed" else np.sort(d)[::-1] if order == "large ones first" else np.sort(d)
            case.dv[pages, h] = d.astype(np.float32)
    # codes of -1, 0 and 1: an output is at most 2^128
    case.v[:] = np.where(case.v == 0x80, 0x80, (case.rng.integers(-1, 2, case.v.shape) & 0xFF)).astype(np.uint8)
    check(case, kv * group)


@pytest.mark.parametrize("kv,group,dim,block,new,lens", SHAPES)
def test_scores_far_apart_where_scales_are(kv, group, dim, block, new, lens):
    """Keys whose scores are hundreds above others', under scales that are as far below the others': either may decide a row."""
    case = Case("e4m3", kv, dim, block, new, lens, seed=6).fill(lens, scale_k=12.0)
    held = np.isfinite(case.dv)
    case.dv[held] = np.exp2(case.rng.choice([-59.0, -20.0, 60.0, 110.0], case.dv.shape))[held].astype(np.float32)
    check(case, kv * group)


@pytest.mark.parametrize("kv,group,dim,block,new,lens", SHAPES)
@pytest.mark.parametrize("fmt", ["int8", "e5m2"])
def test_scales_of_keys_below_the_least_count_as_zero(kv, group, dim, block, new, lens, fmt):
    """Queries so large that keys of 2^-60 give scores of a few units: those below that are keys of zeros, others are not."""
    case = Case(fmt, kv, dim, block, new, lens, seed=7).fill(lens)
    held = np.isfinite(case.dk)
    top = {"int8": 127.0, "e5m2": 57344.0}[fmt]
    case.dk[held] = np.exp2(case.rng.choice([-62.0, -60.5, -60.0, -59.5], case.dk.shape))[held].astype(np.float32)
    check(case, kv * group, q_scale=2.0 ** 61 / top, scale=2 * dim ** -0.5)


@pytest.mark.parametrize("kv,group,dim,block,new,lens", SHAPES)
def test_rows_done_again_are_the_same_captured_on_another_stream_and_beside_others(kv, group, dim, block, new, lens):
    """The same bits every time, without the log-sum-exp, into wider rows; rows of sequences whose scales are small keep theirs."""
    case = Case("int8", kv, dim, block, new, lens, seed=8).fill(lens)
    q, qd = case.queries(kv * group)
    ordinary, _ = qm.qm_cache_attention(qd, **case.device())
    case.dv[case.tables[0, :-(-lens[0] // block)]] *= np.float32(2.0 ** 100)
    d = case.device()
    first, lse = qm.qm_cache_attention(qd, **d, want_lse=True)
    rest = slice(new[0], None)
    assert torch.isfinite(first).all() and first[:new[0]].abs().max() > 1e20
    off = (first[rest].float() - ordinary[rest].float()).abs()          # (one of these may share its thread block: two roundings, and the weights' 11 bits)
    most = max(float(np.nanmax(case.dv[case.tables[b, :-(-n // block)]])) for b, n in enumerate(lens) if b) * 127
    assert (off <= 2.0 ** -7 * 1.01 * ordinary[rest].float().abs() + 4 * 2.0 ** -11 * most).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = qm.qm_cache_attention(qd, **d, want_lse=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(first, other[0]) and torch.equal(lse, other[1])
    wide = torch.full((case.tokens, kv * group + 2, dim), 5.0, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qm.qm_cache_attention(qd, **d, out=wide[:, 1:-1])
    for _ in range(2):
        wide[:, 1:-1] = 0.0
        graph.replay()
        assert torch.equal(wide[:, 1:-1], first) and (wide[:, 0] == 5.0).all() and (wide[:, -1] == 5.0).all()


def test_oracle_counts_least_scales_as_zero():
    codes = np.arange(1, 17, dtype=np.uint8).reshape(1, 1, 16, 1).repeat(16, 3)
    one, low, q = np.ones((1, 1), np.float32), np.full((1, 1), 2.0 ** -61, np.float32), np.full((1, 1, 16), 2.0 ** 60, np.float32)
    out, lse, _ = blocks.cache_attention(q, codes, low, codes, one, np.array([[0]]), [16], [0, 1], "int8", 1.0)
    assert np.allclose(out, 8.5) and np.allclose(lse, np.log(16))
