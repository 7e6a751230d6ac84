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


def reference(g, act):
    """act(g), t of its quotient g / (1 + exp(-t)) and Phi(-|g|), in 64 bits."""
    t = g if act == "silu" else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
    phi = 0.5 * np.array([layer.math.erfc(abs(v) / 2 ** 0.5) for v in g])
    return layer.activation(g, act), np.abs(t), phi


def stated(g, act, dt):
    """What include/qm.h allows act(g) to be off by, in fp32."""
    a, t, phi = reference(g, act)
    if act == "gelu":
        return a, U * (np.abs(g) * phi * (1.2 * g * g + 22) + np.abs(a)) + 2.0 ** -125
    if dt is torch.float32:
        off = 12 if act == "silu" else 6 * t + 12
    else:
        off = (1.3 if act == "silu" else 7.3) * t + 24
    return a, U * off * np.abs(a) + 2.0 ** -139


def check(gates, act, dt, M=3, K=16):
    gates = gates.float()
    h = gated(gates, torch.ones(len(gates)), act, dt, M, K)
    a, off = stated(gates.double().numpy(), act, dt)
    if dt is torch.bfloat16:                                         # rounded once more: half a step, a subnormal one at least
        off = off + np.maximum(2.0 ** -8 * (np.abs(a) + off), 2.0 ** -134)
    bad = np.abs(h - a) > off
    assert not bad.any(), (gates[bad][:5], h[bad][:5], a[bad][:5], (np.abs(h - a) / off)[bad].max())


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act,lo,hi", [("silu", -105, -80), ("gelu_tanh", -11.5, -9), ("gelu", -14.5, -12)])
def test_gates_whose_activation_nears_the_end_of_fp32(act, lo, hi, dt):
    """As long as act(g) is a normal number of fp32 it is there, although exp(-g) is not."""
    check(torch.linspace(lo, hi, 8000, dtype=torch.float64), act, dt)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ACTS)
def test_tiny_and_huge_gates(act, dt):
    """act(g) is g / 2 next to zero and g, or nothing, far from it, with all of fp32's bits."""
    size = 10.0 ** torch.linspace(-37.9, 38.4, 4000, dtype=torch.float64)
    check(torch.cat([size, -size]), act, dt)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K", KERNELS)
def test_ordinary_gates_stay_within_the_stated_bounds(act, M, K, dt):
    """Densely from -16 to 16, and for the quotients as far as they are normal numbers."""
    gates = torch.linspace(-16, 16, 12001, dtype=torch.float64)
    if act == "silu":
        gates = torch.cat([gates, torch.linspace(-88, 88, 12000, dtype=torch.float64)])
    check(gates, act, dt, M, K)
