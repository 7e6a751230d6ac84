"""The activations of qm_gated_linear_int8 over the whole range of gates, each against what the header states.

A gate is made exactly: one code of 1 on either side, and the gate's value as the scale of its weight row."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                                   # half a step of fp32, relative
ACTS = ["silu", "gelu", "gelu_tanh"]
# (rows, codes): one CTA a tile; the contraction split over a cluster; CTA pairs on tiles of 256 rows
KERNELS = [(3, 16), (1, 1024), (2000, 16)]


def gated(gates, ups, act, out_dtype, M=3, K=16):
    """act(gates[j]) * ups[j] in every row -> the M rows as one, which has to be the same for all."""
    N = len(gates)
    one = torch.zeros(max(M, N), K, dtype=torch.uint8)
    one[:, 0] = 1
    x, w = one[:M].cuda(), one[:N].cuda()
    h = qm.qm_gated_linear_int8(x, torch.ones(M, device="cuda"), w, gates.cuda(), w, ups.cuda(), K, act=act, out_dtype=out_dtype)
    bits = h.view(torch.int32 if out_dtype is torch.float32 else torch.int16)
    assert torch.equal(bits, bits[:1].expand_as(bits))
    return h[0].double().cpu().numpy()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K", KERNELS)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_infinite_gates(act, M, K, dt):
    """What the formulas give: +Inf for +Inf, NaN (of 0 times Inf) for -Inf, NaN for NaN; their neighbours as they are without them."""
    inf = float("inf")
    N = 4096
    gates, ups = torch.full((N,), 2.0), torch.full((N,), -0.5)
    clean = gated(gates, ups, act, dt, M, K)
    gates[:4] = torch.tensor([inf, -inf, float("nan"), 3.0e38])
    ups[:4] = torch.tensor([2.0, 2.0, 2.0, 0.5])
    h = gated(gates, ups, act, dt, M, K)
    assert h[0] == inf and np.isnan(h[1]) and np.isnan(h[2])
    assert abs(h[3] / 1.5e38 - 1) <= 2.0 ** -8
    assert np.array_equal(h[4:], clean[4:])
