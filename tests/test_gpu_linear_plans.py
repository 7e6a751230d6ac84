"""qm_linear_int8 and qm_gated_linear_int8 in every way that they are cut, against one another and at the ends of their range."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import layer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                                   # half a step of fp32, relative


def codes(rows, K, seed, low=-127):
    c = np.random.default_rng(seed).integers(low, 128, size=(rows, qm.qm_code_ld(K)), dtype=np.int8)
    return c, torch.from_numpy(c).view(torch.uint8).cuda()


# 1000 weight rows of 4096 codes, 148 SMs.  Rows of x: (rows a tile, parts of the contraction), or the CTA pairs' kernel
# 1: (16, 8); 17: (32, 8); 33: (16, 4); 65: (32, 4); 129: (64, 4); 257: (64, 2); 520: (32, 1); 580: (64, 1); 1160: (128, 1), gated pairs;
# 2320: pairs
CUTS = [1, 17, 33, 65, 129, 257, 520, 580, 1160]


@pytest.mark.parametrize("form", ["plain", "fp32 bias", "bf16 bias", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_the_same_bits_in_every_cut(form, dt):
    """A row's outputs are the same bits in any batch, whichever kernel, tile and split the batch brings with it."""
    N, K, most = 1000, 4096, 2320
    _, x = codes(most, K, 1)
    _, w = codes(N, K, 2)
    _, u = codes(N, K, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    # gates of a few units: sums of K products of codes are some 127^2 / 3 sqrt(K)
    dx = (torch.rand(most, device="cuda", generator=g) + 0.5) * 0.01
    dw, du = ((torch.rand(N, device="cuda", generator=g) + 0.5) * 300 / (127 * 127 / 3 * K ** 0.5) for _ in range(2))
    bias = torch.randn(N, device="cuda", generator=g)

    def call(M):
        if form in ("silu", "gelu", "gelu_tanh"):
            return qm.qm_gated_linear_int8(x[:M], dx[:M], w, dw, u, du, K, act=form, out_dtype=dt)
        b = None if form == "plain" else bias if form == "fp32 bias" else bias.bfloat16()
        return qm.qm_linear_int8(x[:M], dx[:M], w, dw, K, bias=b, out_dtype=dt)
    whole = call(most)
    for M in CUTS:
        assert torch.equal(call(M), whole[:M]), M


@pytest.mark.parametrize("K", [131071, 100000])
def test_longest_contraction_of_cta_pairs(K):
    """Sums up to 2^31 - 2^14 in magnitude in the kernel for many rows."""
    M, N = 1600, 1472
    cx, x = codes(M, K, 5, low=-128)
    cw, w = codes(N, K, 6, low=-128)
    rows, cols = [0, 1, 255, 256, 700, 1599], [0, 1, 127, 128, 300, 1471]
    x[0] = 128; w[0] = 128; w[1] = 127                               # all -128: the largest sum; the other sign
    cx[0] = -128; cw[0] = -128; cw[1] = 127
    y = qm.qm_linear_int8(x, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), K, out_dtype=torch.float32)
    p = layer.product_int8(cx[rows, :K], np.ones(len(rows)), cw[cols, :K], np.ones(len(cols)))
    assert p.max() == 128 * 128 * K
    got = y[rows][:, cols].double().cpu().numpy()
    assert (np.abs(got - p) <= U * np.abs(p)).all()                  # the int32 sum to fp32: half a step


def test_first_call_under_capture_and_from_two_threads():
    """A process whose first products and norms are captured into a graph, and one whose first ones come from two threads at once."""
    import subprocess
    import sys
    code = """
import threading, torch
import paper_2408_02897_b200 as qm
threads = {threads}
x = torch.randint(-127, 128, (300, 256), device="cuda", dtype=torch.int8).view(torch.uint8)
w = torch.randint(-127, 128, (400, 256), device="cuda", dtype=torch.int8).view(torch.uint8)
dx, dw = torch.rand(300, device="cuda") * 1e-2, torch.rand(400, device="cuda") * 1e-2
z, one = torch.randn(300, 256, device="cuda"), torch.ones(256, device="cuda")
big = x[:1].expand(2600, 256).contiguous()
dbig, wide = torch.rand(2600, device="cuda"), w[:1].expand(2600, 256).contiguous()
torch.cuda.synchronize()
def work(stream=None):
    return [qm.qm_linear_int8(x, dx, w, dw, 256, stream=stream), qm.qm_gated_linear_int8(x, dx, w, dw, w, dw, 256, stream=stream),
            qm.qm_linear_int8(big, dbig, wide, dbig, 256, stream=stream), *qm.qm_rms_norm_quantize(z, one, 1e-6, "int8", stream=stream)[:2]]
if threads:
    got = [None, None]
    def run(i, s):
        got[i] = [work(s) for _ in range(20)][-1]
    ts = [threading.Thread(target=run, args=(i, torch.cuda.Stream())) for i in range(2)]
    [t.start() for t in ts]; [t.join() for t in ts]
else:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    graph.replay()
    got = [out]
torch.cuda.synchronize()
want = work()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
"""
    for threads in (False, True):
        r = subprocess.run([sys.executable, "-c", code.format(threads=threads)], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]


@pytest.fixture
def starved_producer():
    L = qm.lib()
    L.qm_debug_set_wait_limit_ns(2_000_000)                            # 2 ms instead of 1 s
    yield L
    L.qm_debug_stop_producer_after(0xffffffff)
    L.qm_debug_set_wait_limit_ns(0)


# (on 148 SMs) one row, and 40, split eight ways over a cluster; 200 rows, one CTA a tile; CTA pairs with a tile each, plain and gated; pairs
# with two tiles, gated three
@pytest.mark.parametrize("M,N,K", [(1, 1000, 8192), (40, 256, 8192), (200, 6000, 384), (257, 7680, 128), (400, 2816, 1024), (600, 9000, 512)])
@pytest.mark.parametrize("stop_after", [0, 1, 2])
@pytest.mark.parametrize("gated", [False, True])
def test_a_kernel_that_gave_up_frees_its_tensor_memory(starved_producer, M, N, K, stop_after, gated):
    """Many calls that give up one after the other, on two streams: each returns, and a full one behind them is right."""
    _, x = codes(M, K, 7)
    _, w = codes(N, K, 8)
    dx, dw = torch.full((M,), 0.01, device="cuda"), torch.full((N,), 0.0001, device="cuda")

    def call(stream=None):
        return qm.qm_gated_linear_int8(x, dx, w, dw, w, dw, K, stream=stream) if gated else qm.qm_linear_int8(x, dx, w, dw, K, stream=stream)
    want = call()
    torch.cuda.synchronize()
    starved_producer.qm_debug_stop_producer_after(stop_after)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [call(streams[i % 2]) for i in range(8)]
    torch.cuda.synchronize()
    for y in got:
        bad = y.isnan()
        assert torch.equal(y[~bad], want[~bad]) and (stop_after or bad.all())
    starved_producer.qm_debug_stop_producer_after(0xffffffff)
    assert torch.equal(call(), want)
