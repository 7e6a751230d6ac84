"""A feed-forward block in 8 bits as a program runs it: norm with the residual, gated product, its codes, down product, the next
norm; eagerly, on a stream of its own, and captured and replayed."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import layer

pytestmark = pytest.mark.gpu

H, F = 320, 704
U = 2.0 ** -24


class Block:
    """Weights quantized once with qm_quantize, a scale per output channel."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.norm = (1 + 0.1 * torch.randn(H, generator=g)).bfloat16().cuda()
        self.w = {}
        for name, shape in (("gate", (H, F)), ("up", (H, F)), ("down", (F, H))):
            w = (torch.randn(shape, generator=g) / shape[0] ** 0.5).bfloat16().cuda()
            codes, delta, _, _ = qm.qm_quantize(qm.operand_of(w, -2), "int8", "channel")
            self.w[name] = (codes, delta)

    def __call__(self, x, residual, stream=None):
        codes, delta, z = qm.qm_rms_norm_quantize(x, self.norm, 1e-6, "int8", residual=residual, stream=stream)
        h = qm.qm_gated_linear_int8(codes, delta, *self.w["gate"], *self.w["up"], H, act="silu", stream=stream)
        hc, hd, _, _ = qm.qm_quantize(qm.operand_of(h, -1), "int8", "channel", stream=stream)
        y = qm.qm_linear_int8(hc, hd, *self.w["down"], F, stream=stream)
        return codes, delta, z, h, hc, hd, y


def int8_of(codes, cols):
    return codes.cpu().numpy().view(np.int8)[0, :, :cols]


def check(block, x, residual, got):
    """Each step from what the step before it left, so that a rounding that falls the other way is not carried along."""
    codes, delta, z, h, hc, hd, y = got
    want_z, want_codes, want_delta = layer.rms_norm_quantize(x.float().cpu().numpy(), block.norm.float().cpu().numpy(), 1e-6, "int8",
                                                             residual.float().cpu().numpy(), bf16=True)
    assert np.array_equal(z.float().cpu().numpy(), want_z)
    assert np.array_equal(int8_of(codes, H), want_codes.view(np.int8))
    assert (np.abs(delta.double().cpu().numpy() - want_delta) <= ((H / 64 + 32) / 2 + 6) * U * want_delta).all()
    w = {k: (int8_of(c, H if k != "down" else F), d.cpu().numpy()) for k, (c, d) in block.w.items()}
    cx, dx = int8_of(codes, H), delta.cpu().numpy()
    g, u = layer.product_int8(cx, dx, *w["gate"]), layer.product_int8(cx, dx, *w["up"])
    want = layer.activation(g, "silu") * u
    # bf16's half step, and in fp32 g's error (3 U |g|) through a slope of at most 1.1, exp's ((2 |g| + 16) U) and u's
    tol = np.abs(want) * (1.01 * 2.0 ** -8 + (2 * np.abs(g) + 24) * U) + 3.4 * U * np.abs(g * u)
    assert (np.abs(h.double().cpu().numpy() - want) <= tol).all()
    p = layer.product_int8(int8_of(hc, F), hd.cpu().numpy(), *w["down"])
    assert (np.abs(y.double().cpu().numpy() - p) <= np.abs(p) * 1.01 * (2.0 ** -8 + 3 * U)).all()


def inputs(rows, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(rows, H, generator=g).bfloat16().cuda(), (3 * torch.randn(rows, H, generator=g)).bfloat16().cuda()


@pytest.mark.parametrize("rows", [1, 5, 77, 300])
def test_block(rows):
    block, (x, r) = Block(1), inputs(rows, 2)
    got = block(x, r)
    check(block, x, r, got)
    # the next layer's norm takes the block's output in, in place
    z0 = got[2].clone()
    nxt = qm.qm_rms_norm_quantize(got[6], block.norm, 1e-6, "int8", residual=got[2], residual_out=got[2])
    want_z, want_codes, _ = layer.rms_norm_quantize(got[6].float().cpu().numpy(), block.norm.float().cpu().numpy(), 1e-6, "int8",
                                                    z0.float().cpu().numpy(), bf16=True)
    assert np.array_equal(got[2].float().cpu().numpy(), want_z) and np.array_equal(int8_of(nxt[0], H), want_codes.view(np.int8))


def test_the_same_block_in_other_formats_by_qm_gemm():
    """The norm's FP8 codes are what qm_gemm takes."""
    block, (x, r) = Block(3), inputs(64, 4)
    w = torch.randn(F, H, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    for fmt in ("e4m3", "e5m2"):
        codes, delta, _ = qm.qm_rms_norm_quantize(x, block.norm, 1e-6, fmt, residual=r)
        wc, wd, _, _ = qm.qm_quantize(qm.operand_of(w, -1), fmt, "channel")
        y, _ = qm.qm_gemm(codes, fmt, delta, "channel", wc, fmt, wd, "channel", H)
        z = (x.float() + r.float()).bfloat16().double()
        n = z * block.norm.double() / (z.square().mean(1, keepdim=True) + 1e-6).sqrt()
        want = n @ w.double().t()
        assert (y[0].double() - want).norm() <= {"e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}[fmt] * 2 ** 0.5 * want.norm()


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_on_another_stream(rows):
    block, (x, r) = Block(6), inputs(rows, 7)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a = block(x, r, stream=side)
    side.synchronize()
    check(block, x, r, a)
    with torch.cuda.stream(side):
        b = block(x, r)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_captured_and_replayed(rows):
    block, (x, r) = Block(8), inputs(rows, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x, r)
    torch.cuda.current_stream().wait_stream(side)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    x2, r2 = inputs(rows, 10)
    with torch.cuda.graph(graph):
        out = block(x, r)
    with torch.cuda.graph(second):
        out2 = block(x2, r2)
    for seed in (11, 12):                                            # both on the same GPU, one behind and beside the other
        a, b = inputs(rows, seed)
        x.copy_(a); r.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            second.replay()
        torch.cuda.synchronize()
        check(block, x, r, out)
        check(block, x2, r2, out2)


def test_two_streams_at_once():
    block = Block(13)
    streams = [torch.cuda.Stream() for _ in range(3)]
    ins = [inputs(rows, 14 + rows) for rows in (2, 50, 280)]
    torch.cuda.synchronize()
    got = [[block(x, r, stream=s) for s, (x, r) in zip(streams, ins)] for _ in range(5)]
    torch.cuda.synchronize()
    for round_ in got:
        for (x, r), g in zip(ins, round_):
            check(block, x, r, g)


def test_a_freed_result_is_not_handed_out_while_its_stream_works():
    """Outputs made for another stream belong to it: the memory of a dropped one goes back to that stream alone."""
    block, (x, r) = Block(15), inputs(300, 16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ptr = block(x, r, stream=side)[6].data_ptr()                       # dropped at once
    mine = [torch.empty(300, H, dtype=torch.bfloat16, device="cuda") for _ in range(64)]
    assert all(t.data_ptr() != ptr for t in mine)
    torch.cuda.synchronize()


def test_products_beside_one_another_and_beside_probes():
    """Kernels of several shapes on streams of their own, beside a probe and a stand-alone product, which all hold tensor memory: the
    results are those of the calls one after the other."""
    g = torch.Generator().manual_seed(17)

    def side(rows, K):
        c = torch.randint(-127, 128, (rows, K), generator=g, dtype=torch.int32).to(torch.int8).view(torch.uint8).cuda()
        return c, (torch.rand(rows, generator=g) * 0.01).cuda()
    calls = []
    for M, N, K in ((1, 200, 1024), (3, 128, 128), (16, 1000, 4096), (70, 2000, 512), (128, 300, 2048), (600, 2048, 256), (2000, 1024, 128)):
        x, w, u = side(M, K), side(N, K), side(N, K)
        calls.append(lambda s, x=x, w=w, K=K: qm.qm_linear_int8(*x, *w, K, stream=s))
        calls.append(lambda s, x=x, w=w, u=u, K=K: qm.qm_gated_linear_int8(*x, *w, *u, K, stream=s))
        calls.append(lambda s, x=x, w=w, K=K: qm.qm_gemm(x[0][None], "int8", x[1], "channel", w[0][None], "int8", w[1], "channel", K, stream=s)[0])
    L, R = (torch.randn(n, 512, generator=g).bfloat16().cuda() for n in (700, 900))
    ops = (qm.operand_of(L, -1), qm.operand_of(R, -1))
    plan = qm.ProbePlan(*ops, "int8", "int8", "tensor", "tensor")
    want = [c(None) for c in calls]
    plan.launch(*ops)
    record = plan.result().record()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(6)]
    for turn in range(8):
        got = []
        for i, c in enumerate(calls):
            if i % 3 == 0:
                plan.launch(*ops, stream=streams[0])
            got.append(c(streams[(i + turn) % 6]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert plan.result().record() == record
