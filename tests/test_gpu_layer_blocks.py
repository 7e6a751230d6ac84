"""The operators with a scale for each block as a layer uses them together, and what the binding refuses."""
import numpy as np
import pytest
import torch

import paper_2408_02897_b200 as qm
from oracle import blocks

pytestmark = pytest.mark.gpu

BF16, FP16, U = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


class Layer:
    """Attention of a decoder layer: FP8 projections, an 8-bit cache."""

    def __init__(self, hidden, heads, kv, dim, block, pages, batch, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv, self.dim, self.hidden = heads, kv, dim, hidden
        width = (heads + 2 * kv) * dim
        self.w = [self.weight(torch.randn(width, hidden, generator=g) * hidden ** -0.5), self.weight(torch.randn(hidden, heads * dim, generator=g) * (heads * dim) ** -0.5)]
        shape = (pages, kv, block, dim)
        self.cache = dict(k_codes=torch.zeros(shape, dtype=torch.uint8, device="cuda"), k_delta=torch.zeros(shape[:2], device="cuda"),
                          v_codes=torch.zeros(shape, dtype=torch.uint8, device="cuda"), v_delta=torch.zeros(shape[:2], device="cuda"))
        self.tables = torch.randperm(pages, generator=g).to(torch.int32)[:pages // batch * batch].view(batch, -1).cuda()

    @staticmethod
    def weight(w):
        return qm.qm_quantize_blocks(qm.operand_of(w.bfloat16().cuda(), -1), "e4m3", side=128)

    def __call__(self, x, lens, starts, fmt, keep=None):
        qkv = qm.qm_linear_fp8(*qm.qm_quantize_blocks(qm.operand_of(x, -1), "e4m3"), *self.w[0], self.hidden)
        qkv = qkv.view(len(x), self.heads + 2 * self.kv, self.dim)
        q, k, v = qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv], qkv[:, self.heads + self.kv:]
        qm.qm_cache_append(k, v, **self.cache, tables=self.tables, lens=lens, starts=starts, fmt=fmt)
        o, _ = qm.qm_cache_attention(q, **self.cache, tables=self.tables, lens=lens, starts=starts, fmt=fmt)
        if keep is not None:
            keep += [q, o]
        o = o.view(len(x), -1)
        return qm.qm_linear_fp8(*qm.qm_quantize_blocks(qm.operand_of(o, -1), "e4m3"), *self.w[1], self.heads * self.dim)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_prompt_and_tokens_after_it(fmt):
    layer = Layer(256, 8, 2, 64, 16, 12, 2)
    g = torch.Generator().manual_seed(1)
    lens = np.zeros(2, np.int32)
    for step, new in enumerate([[40, 7], [1, 1], [1, 1], [3, 0], [1, 1]]):
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        lens += np.array(new, np.int32)
        x = torch.randn(sum(new), 256, generator=g).bfloat16().cuda()
        keep = []
        y = layer(x, torch.from_numpy(lens).cuda(), torch.from_numpy(starts).cuda() if new != [1, 1] else None, fmt, keep)
        assert torch.isfinite(y).all() and tuple(y.shape) == (sum(new), 256)
        q, o = keep
        c = {n: t.cpu().numpy() for n, t in layer.cache.items()}
        want, _, top = blocks.cache_attention(q.float().cpu().numpy(), c["k_codes"], c["k_delta"], c["v_codes"], c["v_delta"], layer.tables.cpu().numpy(), lens,
                                              starts, fmt, 64 ** -0.5)
        # scores of a few units in fp32, weights to 11 bits, the output to bf16
        off = np.abs(o.double().cpu().numpy() - want) - (2 * FP16 * top + 1.01 * BF16 * np.abs(want) + 1e-6)
        assert (off <= 0).all(), (step, off.max())
        # the last product of the very codes that it had
        codes, delta = blocks.quantize_blocks(o.float().cpu().numpy().reshape(len(x), -1), "e4m3", 1)
        p, mags = blocks.product(codes, delta, "e4m3", layer.w[1][0].cpu().numpy()[:, :512], layer.w[1][1].cpu().numpy(), "e4m3", 128)
        assert (np.abs(y.double().cpu().numpy() - p) <= (2 * 36 + 6) * U * mags + 1.01 * BF16 * np.abs(p)).all()


def test_a_step_captured_and_replayed_follows_its_inputs():
    layer, again = Layer(128, 4, 4, 32, 32, 8, 2), Layer(128, 4, 4, 32, 32, 8, 2)
    lens = torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    x = torch.randn(2, 128, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    layer(x, lens, None, "int8")                                  # (outside of a capture once; the step below writes the same again)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = layer(x, lens, None, "int8")
    for n in range(1, 70):
        lens.fill_(n)
        x.copy_(torch.randn(2, 128, generator=torch.Generator().manual_seed(n)).bfloat16())
        graph.replay()
        assert torch.equal(y, again(x, lens, None, "int8")), n
    for n, t in layer.cache.items():
        assert torch.equal(t, again.cache[n]), n


def test_two_streams_at_once():
    layers = [Layer(256, 8, 2, 64, 16, 40, 2, seed=s) for s in (0, 1)]
    streams = [torch.cuda.Stream() for _ in layers]
    g = torch.Generator().manual_seed(3)
    xs = [torch.randn(2, 256, generator=g).bfloat16().cuda() for _ in range(30)]
    lens = [torch.tensor([n + 1, n + 1], dtype=torch.int32, device="cuda") for n in range(30)]
    got = [[], []]
    torch.cuda.synchronize()
    for x, n in zip(xs, lens):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(layers[i](x, n, None, "int8"))
    torch.cuda.synchronize()
    for i in range(2):
        alone = Layer(256, 8, 2, 64, 16, 40, 2, seed=i)
        for x, n, y in zip(xs, lens, got[i]):
            assert torch.equal(y, alone(x, n, None, "int8"))


def test_rows_of_no_sequence_stay_as_they_were():
    layer = Layer(128, 4, 2, 64, 16, 8, 2)
    q = torch.randn(6, 4, 64, device="cuda").bfloat16()
    lens, starts = torch.tensor([3, 2], dtype=torch.int32, device="cuda"), torch.tensor([1, 3, 4], dtype=torch.int32, device="cuda")
    out = torch.full((6, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    qm.qm_cache_attention(q, **layer.cache, tables=layer.tables, lens=lens, starts=starts, out=out)
    assert (out[[0, 4, 5]] == 9.0).all() and (out[1:4] == 0).all()


def test_the_binding_refuses():
    layer = Layer(128, 4, 2, 64, 16, 8, 2)
    c, t = layer.cache, layer.tables
    lens = torch.ones(2, dtype=torch.int32, device="cuda")
    q, k = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 64, device="cuda")

    def refused(call):
        with pytest.raises(qm.QmError):
            call()
    att = lambda q=q, tables=t, lens=lens, **kw: qm.qm_cache_attention(q, **{**c, **kw}, tables=tables, lens=lens)  # noqa: E731
    app = lambda k=k, v=k, **kw: qm.qm_cache_append(k, v, **{**c, **kw}, tables=t, lens=lens)  # noqa: E731
    att()
    refused(lambda: att(q=q.float()))
    refused(lambda: att(q=q[:1]))                                 # a token for each sequence
    refused(lambda: att(q=q[:, :3]))                              # heads that are no multiple
    refused(lambda: att(q=q.transpose(0, 1)))
    refused(lambda: att(q=q[:, :, :32]))
    refused(lambda: att(q=q.cpu()))
    refused(lambda: att(lens=lens.long()))
    refused(lambda: att(lens=lens[:1]))
    refused(lambda: att(tables=t.long()))
    refused(lambda: att(k_delta=c["k_delta"][:4]))
    refused(lambda: att(v_codes=c["v_codes"][:, :1]))
    refused(lambda: att(k_codes=c["k_codes"].view(torch.int8)))
    refused(lambda: qm.qm_cache_attention(q, **c, tables=t, lens=lens, out=torch.empty(2, 4, 64, device="cuda")))
    app()
    refused(lambda: app(v=k.bfloat16()))
    refused(lambda: app(k=k[:, :1]))
    refused(lambda: app(k=k.half(), v=k.half()))
    x = torch.zeros(4, 128, device="cuda")
    op = qm.operand_of(x, -1)
    refused(lambda: qm.qm_quantize_blocks(op, "int8"))
    refused(lambda: qm.qm_quantize_blocks(op, "e4m3", side=64))
    refused(lambda: qm.qm_quantize_blocks(qm.operand_of(x.cpu(), -1), "e4m3"))
    refused(lambda: qm.qm_quantize_blocks(qm.operand_of(x.view(2, 2, 128), -1), "e4m3"))
    codes, delta = qm.qm_quantize_blocks(op, "e4m3")
    qm.qm_linear_fp8(codes, delta, codes, delta, 128, side_w=1)
    refused(lambda: qm.qm_linear_fp8(codes, delta, codes, delta, 128))                # a scale for each row, not for 128
    refused(lambda: qm.qm_linear_fp8(codes, delta, codes, delta, 129, side_w=1))
    refused(lambda: qm.qm_linear_fp8(codes, delta, codes, delta, 128, side_w=16))
    refused(lambda: qm.qm_linear_fp8(codes, delta, codes, delta, 128, side_w=1, fmt_x="int8"))
    refused(lambda: qm.qm_linear_fp8(codes, delta, codes, delta, 128, side_w=1, out_dtype=torch.float16))
    refused(lambda: qm.qm_linear_fp8(codes, delta.t(), codes, delta, 128, side_w=1, bias=torch.zeros(3, device="cuda")))
