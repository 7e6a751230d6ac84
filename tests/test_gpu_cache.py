"""qm_cache_append, byte for byte, and qm_cache_attention against 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import blocks
from oracle.formats import decode_table, positive_grid, qmax

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FORMATS = ["int8", "e4m3", "e5m2"]


class Case:
    """A cache whose blocks lie anywhere; what no sequence holds is NaN codes (FP8) under NaN scales, and table entries out of range."""

    def __init__(self, fmt, kv, dim, block, new, lens, seed=0, width=None, spare=3):
        rng = self.rng = np.random.default_rng(seed)
        self.fmt, self.kv, self.dim, self.block = fmt, kv, dim, block
        self.new, self.lens = np.array(new), np.array(lens, np.int32)
        self.starts = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.tokens = int(self.starts[-1])
        need = [-(-max(int(n), 0) // block) for n in lens]
        pages = sum(need) + spare
        self.tables = np.full((len(lens), width or max(need + [1]) + 2), 2 ** 30, np.int32)
        self.tables[:, -1] = -7
        order = list(rng.permutation(pages))
        for b, n in enumerate(need):
            n = min(n, self.tables.shape[1])
            self.tables[b, :n] = [order.pop() for _ in range(n)]
        shape = (pages, kv, block, dim)
        # nothing stored: codes that are no number where the format has some, scales likewise
        junk = {"int8": 0x80, "e4m3": 0x7F, "e5m2": 0x7E}[fmt]
        self.k, self.v = np.full(shape, junk, np.uint8), np.full(shape, junk, np.uint8)
        self.dk, self.dv = np.full(shape[:2], np.nan, np.float32), np.full(shape[:2], np.nan, np.float32)

    def fill(self, upto, scale_k=1.0, scale_v=1.0):
        """Random codes and scales for positions below upto[b] of each sequence."""
        g = len(positive_grid(self.fmt))
        for b, n in enumerate(upto):
            for i in range(-(-int(n) // self.block)):
                if i >= self.tables.shape[1] or not 0 <= self.tables[b, i] < len(self.k):
                    continue
                page, m = self.tables[b, i], min(self.block, int(n) - i * self.block)
                for codes, delta, s in ((self.k, self.dk, scale_k), (self.v, self.dv, scale_v)):
                    x = self.rng.standard_normal((self.kv, m, self.dim)).astype(np.float32)
                    d = (np.abs(x).max((1, 2)) / np.float32(qmax(self.fmt))).astype(np.float32)
                    for h in range(self.kv):
                        codes[page, h, :m] = blocks.quantize(x[h], self.fmt, np.full(m, d[h], np.float32))
                    delta[page] = (d * s * np.exp(0.5 * self.rng.standard_normal(self.kv))).astype(np.float32)
        return self

    def device(self):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return dict(k_codes=t(self.k), k_delta=t(self.dk), v_codes=t(self.v), v_delta=t(self.dv), tables=t(self.tables), lens=t(self.lens),
                    starts=t(self.starts), fmt=self.fmt)

    def queries(self, heads, scale=1.0, pad=0):
        q = torch.from_numpy(self.rng.standard_normal((self.tokens, heads + pad, self.dim)).astype(np.float32) * scale).bfloat16()
        return q[:, :heads], q.cuda()[:, :heads]


def attention_tolerance(case, q, want, top, scale):
    """A score's sum of `dim` exact products: the tensor cores' levels of fp32 truncation, 2 U of its magnitudes for each of the dim + dim / 16
    additions; then four roundings of the exponent x' = x log2 e + log2 dv. exp's relative error is that absolute one, ex2's own is 2^-22, lg2's and the
    reciprocal's 2^-21 together. A weight is rounded to fp16: 2^-11 of it, or below fp16's normal numbers 2^-39 of the largest. Numerator
    and denominator both have them; the sums add 2 U for each of the keys' 16-blocks and joins; the output is rounded once."""
    kmax = np.nanmax(np.abs(case.dk), initial=0.0) * qmax(case.fmt)       # (of a cache that holds nothing, 0: there is no term)
    qn = np.abs(q).max() * case.dim
    x = abs(scale) * qn * kmax
    n = max(int(case.lens.max()), 1)
    score = x * 2 * (case.dim + case.dim // 16) * U
    ex = score + 4 * U * (x * 1.45 + 80)
    rel = 2 * (ex + 2.0 ** -22 + 2.0 ** -21) + 2.0 ** -11 + 2 * (n / 16 + 20) * U
    vmax = np.nanmax(np.abs(case.dv), initial=0.0) * qmax(case.fmt)
    return rel * top + n * 2.0 ** -39 * vmax + (1.01 * 2.0 ** -8 + rel) * np.abs(want) + 1e-30, ex + 2.0 ** -20 + (n / 8 + 40) * U


def run_attention(case, heads, scale=None, pad=0, starts=True, q_scale=1.0):
    q, qd = case.queries(heads, q_scale, pad)
    scale = case.dim ** -0.5 if scale is None else scale
    d = case.device()
    if not starts:
        d["starts"] = None
    out, lse = qm.qm_cache_attention(qd, **d, scale=scale, want_lse=True)
    want, want_lse, top = blocks.cache_attention(q.float().numpy(), case.k, case.dk, case.v, case.dv, case.tables, case.lens, case.starts, case.fmt, scale)
    return q.float().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy(), want, want_lse, top, scale


def check_attention(case, heads, **kw):
    q, out, lse, want, want_lse, top, scale = run_attention(case, heads, **kw)
    tol, tol_lse = attention_tolerance(case, q, want, top, scale)
    assert out.shape == want.shape and np.isfinite(out).all()
    off = np.abs(out - want) - tol
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))
    empty = np.isneginf(want_lse)
    assert np.array_equal(empty, np.isneginf(lse)) and not out[empty].any()
    off = np.abs(lse - want_lse)[~empty] - tol_lse - 2 * U * np.abs(want_lse[~empty])
    assert (off <= 0).all(), off.max()


GEOMETRY = [(1, 1, 16, 16), (2, 1, 64, 32), (1, 3, 128, 64), (3, 4, 80, 16), (2, 8, 96, 128), (1, 16, 48, 256), (4, 2, 112, 32), (1, 40, 64, 64)]


@pytest.mark.parametrize("kv,group,dim,block", GEOMETRY)
@pytest.mark.parametrize("fmt", FORMATS)
def test_a_token_at_a_time(kv, group, dim, block, fmt):
    lens = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 511, 1000]
    case = Case(fmt, kv, dim, block, [1] * len(lens), lens, seed=dim).fill(lens)
    check_attention(case, kv * group)
    check_attention(case, kv * group, starts=False, pad=3)


@pytest.mark.parametrize("kv,group,dim,block", GEOMETRY)
@pytest.mark.parametrize("fmt", FORMATS)
def test_several_new_tokens(kv, group, dim, block, fmt):
    new = [1, 0, 5, 16, 17, 33, 2, 40, 0]
    lens = [70, 10, 5, 100, 17, 250, 700, 41, 0]
    check_attention(Case(fmt, kv, dim, block, new, lens, seed=block).fill(lens), kv * group)


@pytest.mark.parametrize("new,length", [(130, 130), (257, 300), (128, 1000), (300, 2000)])
@pytest.mark.parametrize("fmt,dim", [("int8", 64), ("e4m3", 128), ("e5m2", 96)])
def test_prompts(new, length, fmt, dim):
    check_attention(Case(fmt, 1, dim, 64, [new, 3], [length, 77], seed=new).fill([length, 77]), 4)


@pytest.mark.parametrize("fmt", FORMATS)
def test_one_long_sequence(fmt):
    lens = [20011]
    check_attention(Case(fmt, 1, 128, 64, [1], lens, seed=5).fill(lens), 4)
    check_attention(Case(fmt, 2, 64, 128, [2], lens, seed=6).fill(lens), 2)


def test_many_sequences():
    """More than the threads that look for a share's beginning; many of them with nothing new or nothing at all."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 60, 700)
    new = np.minimum(rng.integers(0, 3, 700), lens)
    check_attention(Case("int8", 2, 64, 16, new, lens, seed=8).fill(lens), 2)


@pytest.mark.parametrize("new,lens", [([5], [3]), ([4, 1], [0, 9]), ([40, 20], [10, 0]), ([1, 1], [0, 0])])
def test_positions_below_zero_see_nothing(new, lens):
    case = Case("e4m3", 2, 64, 16, new, lens, seed=1).fill(lens)
    check_attention(case, 4)


@pytest.mark.parametrize("scale", [0.0, 3.0, -2.0, 1e-30, 40.0])
def test_scales_of_the_scores(scale):
    lens = [1, 40, 333, 1200]
    case = Case("int8", 2, 64, 32, [1, 2, 1, 1], lens, seed=4).fill(lens, scale_k=0.3)
    check_attention(case, 4, scale=scale)


@pytest.mark.parametrize("q_scale", [1e-30, 1e-3, 3e4, 1e30])
def test_queries_of_any_magnitude(q_scale):
    lens = [50, 333]
    case = Case("e5m2", 2, 128, 32, [1, 2], lens, seed=4).fill(lens)
    check_attention(case, 4, scale=0.1 / q_scale, q_scale=q_scale)


@pytest.mark.parametrize("dim", [64, 128])
def test_values_of_blocks_far_apart_in_scale(dim):
    """Scales of the values from 0 and next to nothing to 10^20: neither numerator nor denominator loses a block."""
    lens = [500, 129, 31, 64]
    case = Case("e4m3", 2, dim, 16, [1, 3, 1, 1], lens, seed=9).fill(lens)
    spread = np.exp(case.rng.uniform(-30, 30, case.dv.shape)).astype(np.float32)
    for kind in range(3):
        c = Case("e4m3", 2, dim, 16, [1, 3, 1, 1], lens, seed=9).fill(lens)
        held = np.isfinite(c.dv)
        c.dv[held] = (c.dv * spread)[held] if kind == 0 else 0.0 if kind == 1 else np.where(c.rng.random(c.dv.shape) < 0.5, 0.0, c.dv)[held]
        check_attention(c, 4)


def test_nan_stays_with_those_who_see_it():
    lens, new = [100, 64, 40], [30, 2, 40]
    case = Case("int8", 2, 64, 16, new, lens, seed=2).fill(lens)
    sound = run_attention(case, 4)[1]
    bad = Case("int8", 2, 64, 16, new, lens, seed=2).fill(lens)
    page = bad.tables[0, 5]                                       # positions 80 .. 95 of sequence 0, head 1
    bad.dv[page, 1] = np.nan
    bad.v[page, 1] = 0
    bad.dk[bad.tables[2, 1], 0] = np.nan                          # positions 16 .. 31 of sequence 2, head 0
    out = run_attention(bad, 4)[1]
    sees = np.zeros(out.shape[:2], bool)
    sees[10:30, 2:] = True                                        # tokens at 80 and later, query heads of head 1
    sees[32 + 16:, :2] = True
    assert np.array_equal(np.isnan(out).all(2), sees) and np.array_equal(np.isnan(out).any(2), sees)
    assert np.array_equal(out[~sees], sound[~sees])


def test_bad_blocks_give_nan_and_are_not_read():
    lens, new = [100, 64, 200], [1, 1, 1]
    case = Case("int8", 2, 64, 16, new, lens, seed=2, width=9).fill([100, 64, 144])
    case.tables[0, 3] = len(case.k)                                # one past the last
    case.tables[1, 0] = -1
    out = run_attention(case, 4)[1]
    assert np.isnan(out).all()                                    # the third is longer than its table


def test_rows_of_starts_out_of_range_are_no_tokens():
    case = Case("int8", 1, 64, 16, [1, 1, 1], [30, 30, 30]).fill([30, 30, 30])
    q, qd = case.queries(2)
    for starts in ([0, 1, 2, 4], [0, 1, -5, 3], [-1, 1, 2, 3], [0, 2, 1, 3]):
        d = case.device()
        d["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        out = torch.full((3, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        qm.qm_cache_attention(qd, **d, out=out)
        k = torch.ones(3, 1, 64, device="cuda")
        qm.qm_cache_append(k, k, **d)
        for b in range(3):
            fits = 0 <= starts[b] <= starts[b + 1] <= 3
            if not fits:
                page = case.tables[b, 1]
                assert np.array_equal(d["k_codes"][page].cpu().numpy(), case.k[page])


def test_rows_of_wider_tensors_and_what_lies_behind():
    lens, new = [40, 100], [2, 3]
    case = Case("e4m3", 2, 64, 32, new, lens, seed=1).fill(lens)
    q, qd = case.queries(4, pad=4)
    whole, _ = qm.qm_cache_attention(qd.contiguous(), **case.device())
    wide = torch.full((9, 7, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    out = wide[2:7, 1:5]
    got, none = qm.qm_cache_attention(qd, **case.device(), out=out)
    assert got is out and none is None and torch.equal(out, whole)
    wide[2:7, 1:5] = 5.0
    assert (wide == 5.0).all()


def test_the_same_bits_every_time_captured_and_on_another_stream():
    lens, new = [4000, 30, 777], [1, 4, 1]
    case = Case("int8", 4, 128, 64, new, lens, seed=1).fill(lens)
    q, qd = case.queries(16)
    d = case.device()
    first, lse = qm.qm_cache_attention(qd, **d, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = qm.qm_cache_attention(qd, **d, want_lse=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(first, other[0]) and torch.equal(lse, other[1])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = qm.qm_cache_attention(qd, **d, want_lse=True)
        graphs.append((g, r))
    for g, r in graphs + graphs:
        g.replay()
        assert torch.equal(first, r[0]) and torch.equal(lse, r[1])
    # a graph follows lengths and tables that change
    d["lens"].copy_(torch.tensor([3999, 30, 700], device="cuda"))
    graphs[0][0].replay()
    assert torch.equal(graphs[0][1][0], qm.qm_cache_attention(qd, **d)[0]) and not torch.equal(graphs[0][1][0], first)


# ------------------------------------------------------------------------------------ append
def run_append(case, dtype, scale=1.0, x=None):
    k, v = (torch.from_numpy(case.rng.standard_normal((case.tokens, case.kv + 2, case.dim)).astype(np.float32) * scale).to(dtype) for _ in range(2)) if x is None else x
    d = case.device()
    qm.qm_cache_append(k.cuda()[:, 1:case.kv + 1], v.cuda()[:, 1:case.kv + 1], **d)
    for x, codes, delta in ((k, case.k, case.dk), (v, case.v, case.dv)):
        blocks.cache_append(x[:, 1:case.kv + 1].float().numpy(), codes, delta, case.tables, case.lens, case.starts, case.fmt)
    for name, want in (("k_codes", case.k), ("v_codes", case.v), ("k_delta", case.dk), ("v_delta", case.dv)):
        assert np.array_equal(d[name].cpu().numpy(), want, equal_nan=name.endswith("delta")), name


@pytest.mark.parametrize("kv,dim,block", [(1, 16, 16), (2, 64, 32), (3, 80, 64), (8, 128, 128), (2, 112, 256)])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append(kv, dim, block, fmt, dtype):
    for new, lens in (([1] * 6, [1, 16, 17, 33, 100, 256]), ([300, 1, 0, 40, 17], [300, 20, 9, 75, 300]), ([2, 3], [500, 3])):
        for scale in (0.1, 10.0):                                 # older codes keep their scale, or are rounded again
            case = Case(fmt, kv, dim, block, new, lens, seed=block).fill(np.array(lens) - np.array(new))
            run_append(case, dtype, scale)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_special_values(fmt):
    new, lens = [3, 40, 20, 5, 2, 20], [3, 40, 30, 9, 40, 20]
    case = Case(fmt, 2, 64, 16, new, lens, seed=1).fill(np.array(lens) - np.array(new))
    k, v = (torch.from_numpy(case.rng.standard_normal((case.tokens, 4, 64)).astype(np.float32)) for _ in range(2))
    k[0:3] = 0.0
    k[1, 1, 3] = -0.0
    k[5, 1, 7] = float("nan")
    v[30, 2, 9] = float("inf")
    v[50:55] *= 1e-30                                              # below the least scale
    k[60:65] *= 1e36
    v[66:68] *= 1e-17
    k[-20:] *= 1e-38
    run_append(case, torch.float32, x=(k, v))


def test_append_twice_is_append_once():
    case = Case("int8", 2, 64, 16, [5, 30], [40, 37], seed=1).fill([35, 7])
    d = case.device()
    k = torch.randn(35, 2, 64, device="cuda") * 3
    qm.qm_cache_append(k, -k, **d)
    once = [d[n].clone() for n in ("k_codes", "v_codes", "k_delta", "v_delta")]
    qm.qm_cache_append(k, -k, **d)
    assert all(torch.equal(a.view(torch.uint8), d[n].view(torch.uint8)) for a, n in zip(once, ("k_codes", "v_codes", "k_delta", "v_delta")))


def test_append_leaves_what_has_no_block():
    case = Case("int8", 1, 64, 16, [4, 1, 20], [2, 30, 100], seed=1, width=3).fill([0, 29, 80])
    case.tables[1, 1] = len(case.k)
    run_append(case, torch.float32)


@pytest.mark.parametrize("fmt", FORMATS)
def test_tokens_generated_one_by_one(fmt):
    """A prompt and then tokens one at a time, appended and attended to, against the attention of the very cache that results; and the cache
    stays near what it was given."""
    kv, heads, dim, block, steps = 2, 4, 64, 16, 40
    case = Case(fmt, kv, dim, block, [9, 25], [9, 25], seed=7, spare=0, width=5)
    pages = list(range(10))
    case.tables = np.array([pages[:5], pages[5:]], np.int32)
    for n in ("k", "v"):
        setattr(case, n, np.zeros((10, kv, block, dim), np.uint8))
        setattr(case, "d" + n, np.zeros((10, kv), np.float32))
    d = case.device()
    rng = np.random.default_rng(1)
    given = [[], []]
    lens = np.zeros(2, np.int32)
    for step in range(steps):
        new = [9, 25] if step == 0 else [1, 1]
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        k, v, q = (torch.from_numpy(rng.standard_normal((sum(new), h, dim)).astype(np.float32)).bfloat16() for h in (kv, kv, heads))
        lens += np.array(new, np.int32)
        d["lens"].copy_(torch.from_numpy(lens))
        d["starts"] = torch.from_numpy(starts).cuda() if step == 0 else None
        qm.qm_cache_append(k.cuda(), v.cuda(), **d)
        out, _ = qm.qm_cache_attention(q.cuda(), **d)
        for b in range(2):
            given[b].append(v[starts[b]:starts[b + 1]].float().numpy())
        if step in (0, 7, 39):
            case.k, case.v = d["k_codes"].cpu().numpy(), d["v_codes"].cpu().numpy()
            case.dk, case.dv = d["k_delta"].cpu().numpy(), d["v_delta"].cpu().numpy()
            case.lens, case.starts = lens, starts
            want, _, top = blocks.cache_attention(q.float().numpy(), case.k, case.dk, case.v, case.dv, case.tables, lens, starts, fmt, dim ** -0.5)
            tol, _ = attention_tolerance(case, q.float().numpy(), want, top, dim ** -0.5)
            assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    table = decode_table(fmt)
    for b in range(2):
        held = np.concatenate([table[case.v[p]] * case.dv[p][:, None, None] for p in case.tables[b]], 1)[:, :lens[b]].transpose(1, 0, 2)
        x = np.concatenate(given[b])
        # a rounding is off by half a step: of int8 half a scale, of FP8 half a step of the value or of the least normal one; rounded again a few times
        step = {"int8": 0.5 * case.dv.max(), "e4m3": 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * case.dv.max(), "e5m2": 2.0 ** -3 * np.abs(x) + 2.0 ** -17 * case.dv.max()}[fmt]
        assert (np.abs(held - x) <= 6 * step).all() and math.isfinite(float(np.abs(held).max()))


# Sequences of 64 query rows of a cached head and more, in calls with many of them (the kernel for 128 rows at a time), beside shorter ones.
TILED = [(16, 2, 64, 16), (20, 1, 128, 64), (16, 3, 80, 32), (24, 4, 48, 128), (17, 8, 96, 256)]


@pytest.mark.parametrize("kv,group,dim,block", TILED)
@pytest.mark.parametrize("fmt", FORMATS)
def test_tiles(kv, group, dim, block, fmt):
    new = [130, 1, 0, 257, 64, 7, 40]
    lens = [130, 300, 9, 400, 65, 100, 39]                        # (of the last one, a token lies below position 0)
    check_attention(Case(fmt, kv, dim, block, new, lens, seed=block + dim).fill(lens), kv * group)


@pytest.mark.parametrize("fmt", FORMATS)
def test_tiles_of_values_far_apart_in_scale(fmt):
    lens, new = [300, 150], [200, 100]
    case = Case(fmt, 16, 64, 16, new, lens, seed=3).fill(lens)
    held = np.isfinite(case.dv)
    spread = np.exp(case.rng.uniform(-25, 25, case.dv.shape)) * (case.rng.random(case.dv.shape) < 0.8)
    case.dv[held] = (case.dv * spread)[held].astype(np.float32)
    check_attention(case, 32)


def test_tiles_nan_and_bad_blocks():
    lens, new = [200, 180], [200, 180]
    case = Case("int8", 16, 64, 16, new, lens, seed=2).fill(lens)
    sound = run_attention(case, 32)[1]
    bad = Case("int8", 16, 64, 16, new, lens, seed=2).fill(lens)
    page = bad.tables[0, 5]                                       # positions 80 .. 95 of sequence 0, head 1
    bad.dv[page, 1] = np.nan
    bad.v[page, 1] = 0
    bad.tables[1, 2] = len(bad.k)                                 # positions 32 .. 47 of sequence 1
    out = run_attention(bad, 32)[1]
    sees = np.zeros(out.shape[:2], bool)
    sees[80:200, 2:4] = True
    sees[200 + 32:] = True
    assert np.array_equal(np.isnan(out).all(2), sees) and np.array_equal(np.isnan(out).any(2), sees)
    assert np.array_equal(out[~sees], sound[~sees])


@pytest.mark.parametrize("fmt,dim", [("int8", 64), ("e4m3", 128), ("e5m2", 80)])
def test_one_sequence_of_several_tokens_among_many_of_one(fmt, dim):
    """The form for eight query rows, and a sequence that has more than one such lot."""
    new, lens = [20] + [1] * 15 + [9], [33] + [50 * i + 1 for i in range(15)] + [700]
    check_attention(Case(fmt, 2, dim, 32, new, lens, seed=dim).fill(lens), 4)


@pytest.mark.parametrize("tokens,kv", [(3, 2), (128, 32)])           # both kernels
def test_lengths_beyond_the_table(tokens, kv):
    """A table of three blocks and a sequence far longer: NaN for whoever sees past it, what is within it as ever, and no time spent on the rest."""
    case = Case("int8", kv, 64, 16, [tokens, 1], [48, 40], seed=1, width=3)
    case.tables[0] = range(3)
    case.tables[1] = range(3, 6)
    d = case.fill([48, 40]).device()
    d["lens"][0] = 2 ** 30
    q = torch.randn(tokens + 1, kv, 64, device="cuda").bfloat16()
    out, _ = qm.qm_cache_attention(q, **d)
    assert torch.isnan(out[:tokens]).all() and torch.isfinite(out[tokens]).all()
    # tokens at positions 40 .. : the first eight see nothing but the table's 48
    d["lens"][0] = 40 + tokens
    out, _ = qm.qm_cache_attention(q, **d)
    inside = min(tokens, 8)
    assert torch.isfinite(out[:inside]).all() and torch.isnan(out[inside:tokens]).all() and torch.isfinite(out[tokens]).all()
