"""Scales of the operators with a scale for each block are taken in their own order alone."""
import pytest
import torch

import paper_2408_02897_b200 as qm

pytestmark = pytest.mark.gpu


def refused(call):
    with pytest.raises(qm.QmError):
        call()


def test_scales_of_a_product():
    x, w = torch.randn(40, 384, device="cuda"), torch.randn(200, 384, device="cuda")
    op = lambda t: qm.operand_of(t, -1)  # noqa: E731
    for side in (1, 128):
        cx, dx = qm.qm_quantize_blocks(op(x), "e4m3")
        cw, dw = qm.qm_quantize_blocks(op(w), "e4m3", side=side)
        assert tuple(dx.shape) == (3, 40) and tuple(dw.shape) == (3, 200 if side == 1 else 2)
        y = qm.qm_linear_fp8(cx, dx, cw, dw, 384, side_w=side)
        # as many in one dimension, and a dimension of one more, are the same scales
        for a, b in ((dx.flatten(), dw.flatten()), (dx[None], dw[None])):
            assert torch.equal(qm.qm_linear_fp8(cx, a, cw, b, 384, side_w=side), y)
        refused(lambda: qm.qm_linear_fp8(cx, dx.t().contiguous(), cw, dw, 384, side_w=side))
        refused(lambda: qm.qm_linear_fp8(cx, dx, cw, dw.t().contiguous(), 384, side_w=side))
        refused(lambda: qm.qm_linear_fp8(cx, dx.view(4, 30), cw, dw, 384, side_w=side))
    # of one row, or one block of the contraction, there is no other order
    one = qm.qm_quantize_blocks(op(x[:1]), "e4m3")
    y = qm.qm_linear_fp8(*one, cw, dw, 384)
    assert torch.equal(qm.qm_linear_fp8(one[0], one[1].t(), cw, dw, 384), y)
    short = qm.qm_quantize_blocks(op(x[:, :128]), "e4m3")
    y = qm.qm_linear_fp8(*short, *short, 128, side_w=1)
    assert torch.equal(qm.qm_linear_fp8(short[0], short[1].t(), short[0], short[1].view(40), 128, side_w=1), y)


def test_scales_of_a_cache():
    shape = (6, 2, 16, 64)
    codes = [torch.randint(0, 100, shape, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.rand(shape[:2], device="cuda") for _ in range(2)]
    tables, lens = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3), torch.tensor([40, 17], dtype=torch.int32, device="cuda")
    q, k = torch.randn(2, 4, 64, device="cuda").bfloat16(), torch.randn(2, 2, 64, device="cuda")
    att = lambda dk, dv: qm.qm_cache_attention(q, codes[0], dk, codes[1], dv, tables, lens)[0]  # noqa: E731
    app = lambda dk, dv: qm.qm_cache_append(k, k, codes[0], dk, codes[1], dv, tables, lens)  # noqa: E731
    app(*scales)
    y = att(*scales)
    assert torch.equal(att(scales[0].flatten(), scales[1].flatten()), y)
    for call in (att, app):
        before = [t.clone() for t in codes + scales]
        refused(lambda: call(scales[0].t().contiguous(), scales[1]))
        refused(lambda: call(scales[0], scales[1].t().contiguous()))
        refused(lambda: call(scales[0].view(4, 3), scales[1]))
        assert all(torch.equal(a, b) for a, b in zip(before, codes + scales))
