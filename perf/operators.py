"""Operators of a transformer layer whose projections run in 8 bits: their plain forms, and the calls that a user makes.

Three operators that follow one another: a root-mean-square norm that takes in the residual and leaves the codes and
scales of its output (one scale per token); the product of such codes with an INT8 weight that has a scale per output
channel; and the gated form of that product, act(gate) * up, of a feed-forward block.

`listed()` holds the cases that stand for their use, `draw(rng)` gives more of the same ranges.
"""
import math

import torch

own = False            # True: `run` calls this package's kernels; False: the plain forms below

LARGEST = 16384 * 4096 * 1024          # multiply-adds of one product, at most
LARGEST_NORM = 16384 * 4096            # elements of one norm, at most
QMAX = {"int8": 127.0, "e4m3": 448.0, "e5m2": 57344.0}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------- the cases
def _norm(name, rows, cols, dtype, fmt, residual, pad=0):
    return dict(name=name, op="norm", rows=rows, cols=cols, dtype=dtype, fmt=fmt, residual=residual, pad=pad)


def _linear(name, m, n, k, out, bias):
    return dict(name=name, op="linear", m=m, n=n, k=k, out=out, bias=bias)


def _gated(name, m, n, k, out, act):
    return dict(name=name, op="gated", m=m, n=n, k=k, out=out, act=act)


def listed():
    return [
        # One token being generated: the norm ahead of a projection, hidden size of BERT-large.
        _norm("norm 1x1024", 1, 1024, "bf16", "int8", True),
        # A ragged batch of prompts with an odd hidden size, rows of a wider buffer (a slice of it).
        _norm("norm 1037x2050 strided", 1037, 2050, "bf16", "int8", True, pad=6),
        # The residual stream kept in fp32, first norm of a stack (nothing to add yet).
        _norm("norm 4096x4096 fp32", 4096, 4096, "fp32", "e4m3", False),
        # The largest batch of the library's encoder workloads at a wide hidden size.
        _norm("norm 16384x4096", 16384, 4096, "bf16", "int8", True),
        # One token through an up projection of BERT-large's sizes: latency.
        _linear("linear 1x4096x1024", 1, 4096, 1024, "bf16", True),
        # A batch of 64 sequences, a token each, through a wide square projection: the weight is what is read.
        _linear("linear 64x8192x8192", 64, 8192, 8192, "bf16", False),
        # A ragged batch of prompts, extents off every tile edge and odd, fp32 logits-like output.
        _linear("linear 770x2031x1000 fp32", 770, 2031, 1000, "fp32", True),
        # BERT-large FFN1 on 32 x 512 tokens: the largest product.
        _linear("linear 16384x4096x1024", 16384, 4096, 1024, "bf16", True),
        # One token through a gated block.
        _gated("gated 1x4096x1024", 1, 4096, 1024, "bf16", "silu"),
        # A few sequences decoded together through a wide gated block.
        _gated("gated 24x8192x4096", 24, 8192, 4096, "bf16", "gelu_tanh"),
        # A prompt of odd length, odd sizes.
        _gated("gated 333x2730x1025 fp32", 333, 2730, 1025, "fp32", "gelu"),
        # A prefill of 8192 tokens: both projections are LARGEST multiply-adds together.
        _gated("gated 8192x4096x1024", 8192, 4096, 1024, "bf16", "silu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "gated"])
    if op == "norm":
        rows, cols = _log(rng, 1, 16384), _log(rng, 64, 8192)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        cols = cols if rng.random() < 0.4 else max(64, cols // 64 * 64)
        rows = max(1, min(rows, LARGEST_NORM // cols // (2 if dtype == "fp32" else 1)))
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, fmt=rng.choice(["int8", "int8", "e4m3", "e5m2"]),
                    residual=rng.random() < 0.75, pad=rng.choice([0, 0, 8, 5]))
    m, n, k = _log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 64, 8192)
    if rng.random() < 0.6:
        n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
    m = max(1, min(m, LARGEST // (n * k) // (2 if op == "gated" else 1)))
    out = rng.choice(["bf16", "bf16", "fp32"])
    if op == "linear":
        return dict(op=op, m=m, n=n, k=k, out=out, bias=rng.random() < 0.5)
    return dict(op=op, m=m, n=n, k=k, out=out, act=rng.choice(["silu", "gelu", "gelu_tanh"]))


# ------------------------------------------------------------------------------- what a program has in hand
def _codes(rows, cols, std, gen, outliers=False):
    """INT8 codes [rows, cols padded to 16] (the padding zero), as bytes, and the scale of each row."""
    x = torch.randn(rows, cols, device="cuda", generator=gen) * std
    if outliers:                       # a few feature channels stand out, as in activations
        x[:, ::97] *= 8.0
    top = x.abs().amax(1)
    delta = torch.where(top > 0, top / 127.0, torch.ones_like(top))
    codes = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    codes[:, :cols] = torch.round(x / delta[:, None]).clamp_(-127, 127).to(torch.int8)
    return codes.view(torch.uint8), delta


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    if case["op"] == "norm":
        rows, cols, dt = case["rows"], case["cols"], DTYPE[case["dtype"]]

        def wide():
            t = torch.randn(rows, cols + case["pad"], device="cuda", generator=gen)
            t[:, ::97] *= 20.0         # channels that stand out
            return t.to(dt)[:, :cols]
        s["x"] = wide()
        s["residual_in"] = wide() if case["residual"] else None
        s["weight"] = (1.0 + 0.1 * torch.randn(cols, device="cuda", generator=gen)).to(dt)
        s["qmax"] = torch.tensor(QMAX[case["fmt"]], device="cuda")   # on the GPU: divided by, not multiplied with its inverse
        return s
    m, n, k = case["m"], case["n"], case["k"]
    s["cx"], s["dx"] = _codes(m, k, 1.0, gen, outliers=True)
    s["cw"], s["dw"] = _codes(n, k, 0.02, gen)
    if case["op"] == "gated":
        s["cu"], s["du"] = _codes(n, k, 0.02, gen)
    s["b"] = torch.randn(n, device="cuda", generator=gen) * 0.1 if case.get("bias") else None
    return s


# ------------------------------------------------------------------------------- one pass
def _plain_norm(s):
    # z = x + residual, rounded to the stream's type; v = z w; codes are those of v under Eq. 1's scale of its row, and
    # the norm's factor 1 / rms(z) goes into the scale: the codes stand for v / rms(z)
    z = s["x"]
    if s["residual_in"] is not None:
        z = (z.float() + s["residual_in"].float()).to(z.dtype)
    zf = z.float()
    v = zf * s["weight"].float()
    top = v.abs().amax(1, keepdim=True)
    own_delta = torch.where(top > 0, top / s["qmax"], torch.ones_like(top))
    t = v / own_delta
    if s["fmt"] == "int8":
        codes = torch.round(t).clamp_(-127.0, 127.0).to(torch.int8)
    else:
        codes = t.clamp_(-QMAX[s["fmt"]], QMAX[s["fmt"]]).to(FP8[s["fmt"]])
    factor = 1.0 / torch.sqrt(zf.square().mean(1, keepdim=True) + EPS)
    return {"codes": codes, "delta": (own_delta * factor)[:, 0],
            "residual": z if s["residual_in"] is not None else None}


def _plain_product(s, codes, delta):
    k = s["k"]
    acc = s["cx"].view(torch.int8)[:, :k].float() @ codes.view(torch.int8)[:, :k].float().t()
    return acc * (s["dx"][:, None] * delta[None, :])


def _plain_act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    if act == "gelu":
        return 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def run(s):
    if own:
        import paper_2408_02897_b200 as qm
        if s["op"] == "norm":
            codes, delta, residual = qm.qm_rms_norm_quantize(s["x"], s["weight"], EPS, s["fmt"], residual=s["residual_in"])
            held = torch.int8 if s["fmt"] == "int8" else FP8[s["fmt"]]
            return {"codes": codes[0].view(held)[:, :s["cols"]], "delta": delta, "residual": residual}
        if s["op"] == "linear":
            return qm.qm_linear_int8(s["cx"], s["dx"], s["cw"], s["dw"], s["k"], bias=s["b"], out_dtype=DTYPE[s["out"]])
        return qm.qm_gated_linear_int8(s["cx"], s["dx"], s["cw"], s["dw"], s["cu"], s["du"], s["k"], act=s["act"],
                                       out_dtype=DTYPE[s["out"]])
    if s["op"] == "norm":
        return _plain_norm(s)
    if s["op"] == "linear":
        y = _plain_product(s, s["cw"], s["dw"])
        return (y if s["b"] is None else y + s["b"]).to(DTYPE[s["out"]])
    g, u = _plain_product(s, s["cw"], s["dw"]), _plain_product(s, s["cu"], s["du"])
    return (_plain_act(g, s["act"]) * u).to(DTYPE[s["out"]])


# ------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        n, es = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * (es * (3 if case["residual"] else 1) + 1) + case["cols"] * es + 4 * case["rows"], "flops": 6 * n}
    m, n, k, es = case["m"], case["n"], case["k"], 2 if case["out"] == "bf16" else 4
    w = 2 if case["op"] == "gated" else 1
    return {"bytes": m * k + w * n * k + 4 * (m + w * n + (n if case.get("bias") else 0)) + m * n * es, "flops": 2 * w * m * n * k}


# ------------------------------------------------------------------------------- the definition, in 64 bits
def _nearest_fp8(t, fmt):
    """The nearest value of the format's grid, ties to the even code; t is within its range."""
    mantissa, least = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(t.abs().clamp_min(2.0 ** least))[1] - 1            # 2^e <= |t|, at least the smallest normal's
    step = torch.ldexp(torch.ones_like(t), e - mantissa)
    return torch.round(t / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        z = s["x"].double()
        if s["residual_in"] is not None:                               # the stream is held in its type
            z = (z + s["residual_in"].double()).to(s["x"].dtype).double()
        y = z * s["weight"].double() / (z.pow(2).sum(1, keepdim=True) / case["cols"] + EPS).sqrt()
        top = y.abs().max(1, keepdim=True).values
        delta = torch.where(top > 0, top / QMAX[case["fmt"]], torch.ones_like(top))
        codes = torch.round(y / delta).to(torch.int8) if case["fmt"] == "int8" else _nearest_fp8(y / delta, case["fmt"])
        return {"codes": codes, "delta": delta[:, 0], "residual": z if s["residual_in"] is not None else None}

    def product(codes, delta):
        a, b = s["cx"].view(torch.int8).double(), codes.view(torch.int8).double()      # (padding is zero)
        return torch.einsum("ik,jk->ij", a, b) * s["dx"].double()[:, None] * delta.double()[None, :]
    y = product(s["cw"], s["dw"])
    if case["op"] == "linear":
        return y if s["b"] is None else y + s["b"].double()[None, :]
    if case["act"] == "silu":
        y = y * torch.sigmoid(y)
    elif case["act"] == "gelu":
        y = y * torch.special.ndtr(y)
    else:
        y = y * torch.sigmoid(2.0 * (2.0 / math.pi) ** 0.5 * (y + 0.044715 * y ** 3))
    return y * product(s["cu"], s["du"])
