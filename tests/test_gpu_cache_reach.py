"""Lengths beyond a table in the kernel for many query rows, and which calls have it."""
import pytest
import torch

import paper_2408_02897_b200 as qm
from test_gpu_cache import Case, check_attention

pytestmark = pytest.mark.gpu


def launches(call):
    before = qm.kernel_launches()
    out = call()
    return out, qm.kernel_launches() - before


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv,group,tokens", [(16, 4, 256), (64, 1, 200), (64, 4, 300)])
def test_lengths_beyond_the_table_in_tiles(dim, kv, group, tokens):
    """A table of three blocks and a sequence far longer: NaN for whoever sees past it, what is within it as ever, and no time spent on the rest."""
    case = Case("int8", kv, dim, 16, [tokens, 1], [48, 40], seed=1, width=3)
    case.tables[0] = range(3)
    case.tables[1] = range(3, 6)
    d = case.fill([48, 40]).device()
    q = torch.randn(tokens + 1, kv * group, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).bfloat16()
    for length in (2 ** 30, 2 ** 31 - 1):
        d["lens"][0] = length
        (out, _), n = launches(lambda: qm.qm_cache_attention(q, **d))
        assert n == 3                                             # tiles, rows, join
        assert torch.isnan(out[:tokens]).all() and torch.isfinite(out[tokens]).all()
    # the first eight tokens are at positions 40 .. 47 and see nothing but the table's 48
    d["lens"][0] = 40 + tokens
    (out, _), n = launches(lambda: qm.qm_cache_attention(q, **d))
    assert n == 3 and torch.isfinite(out[:8]).all() and torch.isnan(out[8:tokens]).all() and torch.isfinite(out[tokens]).all()
    # the same eight by themselves
    case.lens[:] = [48, 40]
    few = dict(d, lens=torch.tensor([48, 40], dtype=torch.int32, device="cuda"), starts=torch.tensor([0, 8, 9], dtype=torch.int32, device="cuda"))
    alone, _ = qm.qm_cache_attention(torch.cat([q[:8], q[tokens:]]), **few)
    # both rounded to bf16, from weights of 11 bits (of which numerator and denominator have the errors)
    most = float(d["v_delta"].nan_to_num().max()) * 127
    assert ((alone[:8].float() - out[:8].float()).abs() <= 2.0 ** -7 * 1.01 * alone[:8].float().abs() + 4 * 2.0 ** -11 * most).all()


@pytest.mark.parametrize("kv,group,dim,block,new,lens", [
    (1, 3, 128, 64, [1, 1, 1], [300, 300, 300]), (3, 3, 128, 64, [1, 1, 1, 1], [300, 301, 17, 999]), (5, 2, 64, 16, [1, 2, 0, 1, 9], [333, 200, 50, 1000, 77]),
    (8, 4, 128, 32, [1] * 7, [2000, 40, 41, 42, 1999, 33, 1]), (2, 1, 64, 16, [20, 1, 3], [900, 901, 902])])
@pytest.mark.parametrize("fmt", ["int8", "e4m3", "e5m2"])
def test_shares_that_begin_and_end_inside_rows(kv, group, dim, block, new, lens, fmt):
    """Thread blocks' equal shares of keys cross heads and sequences: none is skipped or taken twice (a log-sum-exp would be off by its logarithm)."""
    check_attention(Case(fmt, kv, dim, block, new, lens, seed=kv + dim).fill(lens), kv * group)


def test_a_prompt_among_sequences_without_new_tokens():
    """The rows of a call are one sequence's, however many others there are without any."""
    new, lens = [0] * 150 + [200] + [0] * 149, [5] * 150 + [300] + [33] * 149
    case = Case("int8", 64, 64, 32, new, lens, seed=3).fill(lens)
    q, qd = case.queries(64)
    _, n = launches(lambda: qm.qm_cache_attention(qd, **case.device()))
    assert n == 3
    small = Case("int8", 16, 64, 32, new, lens, seed=3).fill(lens)
    check_attention(small, 64)
