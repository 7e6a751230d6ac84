"""qm_cache_append and qm_cache_attention with entries of `starts` that name no rows, beside sequences whose rows they do name."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import blocks
from test_gpu_cache import Case, attention_tolerance

pytestmark = pytest.mark.gpu

TOP, LOW = 2 ** 31 - 1, -2 ** 31
# starts, tokens, lengths. Rows of the tokens that no sequence has are in some of them.
STARTS = [
    ([0, 300, 600, 0, 0, 0, 0], 600, [500, 301, 9, 40, 0, 7]),                       # what is behind the last sequence is zeros
    ([0, 300, 600, -1, -1, -1, -1, -1], 600, [500, 301, 9, 40, 0, 7, 16]),
    ([0, 1000, 5, 300, -7, 300, 520], 520, [40, 100, 330, 20, 20, 221]),
    ([TOP, 0, 130, LOW, 130, 400], 400, [30, 130, 99, 17, 300]),
    ([3, 200, LOW, 200, 390, 50, -3, 391], 391, [197, 50, 240, 333, 77, 20, 30]),
    ([0, 1, 2, 900, 3, 4], 4, [33, 48, 50, 60, 17]),                                  # a token at a time
]


def case_of(starts, tokens, lens, kv, dim, block, fmt, seed=1):
    """Valid sequences' codes up to their old lengths; and [(b, first row, end)] of those."""
    valid = [(b, starts[b], starts[b + 1]) for b in range(len(lens)) if 0 <= starts[b] < starts[b + 1] <= tokens]
    case = Case(fmt, kv, dim, block, [0] * len(lens), lens, seed=seed)
    case.starts, case.tokens = np.array(starts, np.int64).astype(np.int32), tokens
    return case, valid


@pytest.mark.parametrize("starts,tokens,lens", STARTS)
@pytest.mark.parametrize("kv,dim,block", [(1, 64, 16), (3, 80, 32)])
def test_append(starts, tokens, lens, kv, dim, block):
    case, valid = case_of(starts, tokens, lens, kv, dim, block, "int8")
    new = np.zeros(len(lens), int)
    for b, first, end in valid:
        new[b] = end - first
    case.fill(np.maximum(np.array(lens) - new, 0))
    d = case.device()
    k, v = (torch.from_numpy(case.rng.standard_normal((tokens, kv, dim)).astype(np.float32)) for _ in range(2))
    qm.qm_cache_append(k.cuda(), v.cuda(), **d)
    for x, codes, delta in ((k, case.k, case.dk), (v, case.v, case.dv)):
        for b, first, end in valid:
            blocks.cache_append(x.numpy(), codes, delta, case.tables[b:b + 1], case.lens[b:b + 1], [first, end], "int8")
    for name, want in (("k_codes", case.k), ("v_codes", case.v), ("k_delta", case.dk), ("v_delta", case.dv)):
        assert np.array_equal(d[name].cpu().numpy(), want, equal_nan=name.endswith("delta")), name


@pytest.mark.parametrize("starts,tokens,lens", STARTS)
@pytest.mark.parametrize("kv,group,dim,block", [(1, 2, 64, 16), (16, 2, 64, 32), (32, 4, 128, 16)])      # the last two: tiles, if there are tokens enough
def test_attention(starts, tokens, lens, kv, group, dim, block):
    case, valid = case_of(starts, tokens, lens, kv, dim, block, "int8")
    case.fill(lens)
    q, qd = case.queries(kv * group)
    out = torch.full((tokens, kv * group, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    before = qm.kernel_launches()
    qm.qm_cache_attention(qd, **case.device(), out=out)
    assert qm.kernel_launches() - before == (3 if kv > 1 and tokens >= 130 else 2)      # tiles, rows, join
    q, out, rest = q.float().numpy(), out.double().cpu().numpy(), np.ones(tokens, bool)
    for b, first, end in valid:
        want, _, top = blocks.cache_attention(q, case.k, case.dk, case.v, case.dv, case.tables[b:b + 1], case.lens[b:b + 1], [first, end], "int8", dim ** -0.5)
        tol, _ = attention_tolerance(case, q, want, top, dim ** -0.5)
        rows = slice(first, end)
        assert (np.abs(out - want) <= tol)[rows].all(), b
        rest[rows] = False
    assert (out[rest] == 7.0).all()


def test_append_to_very_many_sequences():
    """More units of work than thread blocks: several to each, of sequences with nothing, one or several tokens and entries that name no rows."""
    rng = np.random.default_rng(4)
    batch, kv, dim, block = 6000, 4, 16, 16
    new = rng.choice([0, 1, 1, 2, 20], batch)
    starts = np.concatenate([[0], np.cumsum(new)])
    tokens = int(starts[-1])
    lens = new + rng.integers(0, 20, batch)
    starts[rng.choice(batch + 1, 300, replace=False)] = -1
    valid = (starts[:-1] >= 0) & (starts[1:] >= starts[:-1]) & (starts[1:] <= tokens)
    case = Case("int8", kv, dim, block, [0] * batch, lens, seed=2)
    case.starts, case.tokens = starts.astype(np.int32), tokens
    for delta in (case.dk, case.dv):
        delta[:] = rng.random(delta.shape).astype(np.float32) * 0.01
    for codes in (case.k, case.v):
        codes[:] = rng.integers(0, 128, codes.shape)
    d = case.device()
    k, v = (torch.from_numpy(rng.standard_normal((tokens, kv, dim)).astype(np.float32)) for _ in range(2))
    qm.qm_cache_append(k.cuda(), v.cuda(), **d)
    for x, codes, delta in ((k, case.k, case.dk), (v, case.v, case.dv)):
        for b in np.flatnonzero(valid):
            blocks.cache_append(x.numpy(), codes, delta, case.tables[b:b + 1], case.lens[b:b + 1], starts[b:b + 2], "int8")
    for name, want in (("k_codes", case.k), ("v_codes", case.v), ("k_delta", case.dk), ("v_delta", case.dv)):
        assert np.array_equal(d[name].cpu().numpy(), want), name
