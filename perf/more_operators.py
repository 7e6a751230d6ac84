"""Operators of a transformer layer held in 8 bits with a scale for each block: their plain forms, and the calls that a user makes.

Two pairs. Codes of a matrix in FP8 with a scale for each 128 entries of the contraction (of one row, or of 128 rows), and the
product of two such matrices, as training runs its forward, input-gradient and weight-gradient products. A cache of keys and
values in 8 bits with a scale for each block of tokens and head, into which new tokens are written, and the attention that reads it,
for a token at a time and for prompts.

`listed()` holds the cases that stand for their use, `draw(rng)` gives more of the same ranges.
"""
import math

import torch

own = False            # True: `run` calls this package's kernels; False: the plain forms below

SIDE = 128                                     # contraction entries, and rows of a weight, under one scale
LARGEST = 16384 * 4096 * 1024                  # multiply-adds of one product, at most
LARGEST_CODES = 16384 * 4096                   # elements of one matrix to be coded, at most
LARGEST_CACHE = 64 * 8192 * 8 * 128            # elements of the keys that one attention reads, at most
LARGEST_SCORES = 32 * 2048 * 4096              # query rows x keys of one attention, at most
QMAX = {"int8": 127.0, "e4m3": 448.0, "e5m2": 57344.0}
HELD = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------- the cases
def _codes_case(name, rows, cols, dtype, fmt, side, strided):
    return dict(name=name, op="codes", rows=rows, cols=cols, dtype=dtype, fmt=fmt, side=side, strided=strided)


def _product(name, m, n, k, fmt_x, fmt_w, side, out, bias):
    return dict(name=name, op="product", m=m, n=n, k=k, fmt_x=fmt_x, fmt_w=fmt_w, side=side, out=out, bias=bias)


def _append(name, batch, most_new, most_old, kv_heads, dim, block, dtype, fmt):
    return dict(name=name, op="append", batch=batch, most_new=most_new, most_old=most_old, kv_heads=kv_heads, dim=dim, block=block,
                dtype=dtype, fmt=fmt)


def _attention(name, batch, most_new, most_len, heads, kv_heads, dim, block, fmt, even=False):
    return dict(name=name, op="attention", batch=batch, most_new=most_new, most_len=most_len, heads=heads, kv_heads=kv_heads, dim=dim,
                block=block, fmt=fmt, even=even)


def listed():
    return [
        # The activations of 32 x 512 tokens ahead of a product: a scale for each 128 of a token's features.
        _codes_case("codes 16384x4096", 16384, 4096, "bf16", "e4m3", 1, False),
        # A weight of BERT-large's FFN in its storage order, contraction strided, for the input gradient: squares of 128.
        _codes_case("codes weight 4096x1024 fp32", 4096, 1024, "fp32", "e4m3", 128, True),
        # One token through an up projection: latency.
        _product("product 1x4096x1024", 1, 4096, 1024, "e4m3", "e4m3", 128, "bf16", True),
        # 64 sequences, a token each, through a wide square projection: the weight is what is read.
        _product("product 64x8192x8192", 64, 8192, 8192, "e4m3", "e4m3", 128, "bf16", False),
        # A ragged batch of prompts, extents off every tile edge and odd; an output gradient in E5M2.
        _product("product 770x2031x1000 fp32", 770, 2031, 1000, "e5m2", "e4m3", 128, "fp32", False),
        # BERT-large FFN1 on 32 x 512 tokens: the largest product.
        _product("product 16384x4096x1024", 16384, 4096, 1024, "e4m3", "e4m3", 128, "bf16", True),
        # Its weight gradient: contraction over the tokens, a scale for each 128 of them on both sides.
        _product("weight gradient 4096x1024x16384", 4096, 1024, 16384, "e5m2", "e4m3", 1, "fp32", False),
        # One token of each of 64 sequences goes into the cache.
        _append("append 64 tokens", 64, 1, 2000, 8, 128, 64, "bf16", "int8"),
        # Prompts of up to 1000 tokens, heads of BERT-large.
        _append("append 8 prompts", 8, 1000, 300, 16, 64, 32, "bf16", "e4m3"),
        # One token of one sequence, heads of BERT-large: latency.
        _attention("attention 1 token on 384", 1, 1, 384, 16, 16, 64, 16, "int8", even=True),
        # One token of each of 64 sequences of any length up to 8192, four query heads to a cached one: the largest cache.
        _attention("attention 64 tokens on 8192", 64, 1, 8192, 32, 8, 128, 64, "int8"),
        # The second half of a prompt of 4096 tokens: the most arithmetic.
        _attention("attention 2048 tokens on 4096", 1, 2048, 4096, 32, 8, 128, 128, "e4m3", even=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["codes", "product", "product", "append", "attention", "attention"])
    if op == "codes":
        rows, cols = _log(rng, 1, 16384), _log(rng, 64, 8192)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        rows = max(1, min(rows, LARGEST_CODES // cols // (2 if dtype == "fp32" else 1)))
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, fmt=rng.choice(["e4m3", "e4m3", "e5m2"]), side=rng.choice([1, 1, 128]),
                    strided=rng.random() < 0.4)
    if op == "product":
        m, n, k = _log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 64, 8192)
        if rng.random() < 0.6:
            n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
        m = max(1, min(m, LARGEST // (n * k)))
        return dict(op=op, m=m, n=n, k=k, fmt_x=rng.choice(["e4m3", "e4m3", "e5m2"]), fmt_w=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    side=rng.choice([128, 128, 1]), out=rng.choice(["bf16", "bf16", "fp32"]), bias=rng.random() < 0.5)
    kv_heads, dim, block = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 64, 80, 96, 128, 128]), rng.choice([16, 32, 64, 128])
    fmt, batch = rng.choice(["int8", "e4m3", "e5m2"]), _log(rng, 1, 64)
    if op == "append":
        new = 1 if rng.random() < 0.5 else max(1, min(_log(rng, 1, 2048), 16384 // batch))
        return dict(op=op, batch=batch, most_new=new, most_old=_log(rng, 1, 2048), kv_heads=kv_heads, dim=dim, block=block,
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), fmt=fmt)
    heads = kv_heads * rng.choice([1, 2, 4, 8])
    length = max(1, min(_log(rng, 16, 8192), LARGEST_CACHE // (batch * kv_heads * dim)))
    new = 1 if rng.random() < 0.6 else max(1, min(_log(rng, 1, 2048), length, LARGEST_SCORES // (batch * heads * length)))
    return dict(op=op, batch=batch, most_new=new, most_len=length, heads=heads, kv_heads=kv_heads, dim=dim, block=block, fmt=fmt,
                even=rng.random() < 0.3)


# ------------------------------------------------------------------------------- what a program has in hand
def _up(n, to):
    return (n + to - 1) // to * to


def _blocked(rows, cols, side, fmt, std, gen):
    """FP8 codes [rows, cols padded to 16] (the padding zero), as bytes, and scales [blocks of the contraction, blocks of rows]."""
    x = torch.randn(rows, cols, device="cuda", generator=gen) * std
    x[:, ::97] *= 8.0                  # a few channels stand out, as in activations
    full = torch.zeros(_up(rows, side), _up(cols, SIDE), device="cuda")
    full[:rows, :cols] = x
    tiles = full.view(full.shape[0] // side, side, full.shape[1] // SIDE, SIDE)
    delta = tiles.abs().amax((1, 3)) / QMAX[fmt]
    delta = torch.where(delta > 0, delta, torch.ones_like(delta))
    codes = (tiles / delta[:, None, :, None]).view(full.shape)[:rows, :_up(cols, 16)].to(HELD[fmt])
    return codes.contiguous().view(torch.uint8), delta.t().contiguous()


def _spread(most, n, gen_cpu, even):
    """n whole numbers from 1 to `most`, the largest among them."""
    v = torch.randint(1, most + 1, (n,), generator=gen_cpu)
    v[int(torch.randint(0, n, (1,), generator=gen_cpu))] = most
    return torch.full((n,), most) if even else v


def _cache(pages, case, gen):
    """Codes [pages, heads, tokens of a block, dim] of a cache that has been written, and the scales of its blocks."""
    shape = (pages, case["kv_heads"], case["block"], case["dim"])
    codes, deltas = [], []
    for keys in (True, False):
        x = torch.randn(shape, device="cuda", generator=gen)
        if keys:
            x[..., ::31] *= 3.0        # channels that stand out
        delta = x.abs().amax((2, 3)) / QMAX[case["fmt"]]
        x = x.div_(delta[:, :, None, None])
        codes.append((x.round_() if case["fmt"] == "int8" else x).to(HELD[case["fmt"]]).view(torch.uint8))
        deltas.append(delta)
    return codes, deltas


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    if case["op"] == "codes":
        x = torch.randn(case["rows"], _up(case["cols"], 8), device="cuda", generator=gen) * 0.02 if not case["strided"] else \
            torch.randn(case["cols"], _up(case["rows"], 8), device="cuda", generator=gen) * 0.02
        x[:, ::97] *= 20.0             # channels that stand out
        x = x.to(DTYPE[case["dtype"]])
        s["x"] = x[:, :case["rows"]].t() if case["strided"] else x[:, :case["cols"]]     # [rows, cols], either order in memory
        s["qmax"] = torch.tensor(QMAX[case["fmt"]], device="cuda")     # on the GPU: divided by, not multiplied with its inverse
        return s
    if case["op"] == "product":
        s["cx"], s["dx"] = _blocked(case["m"], case["k"], 1, case["fmt_x"], 1.0, gen)
        s["cw"], s["dw"] = _blocked(case["n"], case["k"], case["side"], case["fmt_w"], 0.02, gen)
        s["b"] = torch.randn(case["n"], device="cuda", generator=gen) * 0.1 if case["bias"] else None
        return s
    cpu = torch.Generator()
    cpu.manual_seed(seed)
    batch, block = case["batch"], case["block"]
    fixed = torch.Generator()
    fixed.manual_seed(batch + case["most_new"])                        # how many tokens there are is the case's, where they go the seed's
    new = _spread(case["most_new"], batch, fixed, case.get("even", False))
    if case["op"] == "append":
        lens = new + torch.randint(0, case["most_old"] + 1, (batch,), generator=cpu)
    else:
        lens = torch.maximum(new, _spread(case["most_len"], batch, cpu, case["even"]))
    tokens, s["longest"] = int(new.sum()), int(lens.max())
    blocks = (lens + block - 1) // block
    pages = batch * ((case["most_len"] if case["op"] == "attention" else case["most_new"] + case["most_old"]) // block + 1)
    order = torch.randperm(pages, generator=cpu).to(torch.int32)[:int(blocks.sum())]       # blocks of a sequence lie anywhere
    tables = torch.zeros(batch, int(blocks.max()), dtype=torch.int32)
    tables[torch.arange(tables.shape[1])[None, :] < blocks[:, None]] = order
    s["tables"], s["lens"] = tables.cuda(), lens.to(torch.int32).cuda()
    s["starts"] = None                                                 # a token for each sequence
    if case["most_new"] > 1:
        s["starts"] = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).to(torch.int32).cuda()
    (s["kc"], s["vc"]), (s["dk"], s["dv"]) = _cache(pages, case, gen)
    heads = case.get("heads", 0)
    wide = torch.randn(tokens, heads + 2 * case["kv_heads"], case["dim"], device="cuda", generator=gen)     # a fused projection's output
    if case["op"] == "append":
        wide *= torch.exp(0.3 * torch.randn(tokens, 1, 1, device="cuda", generator=gen))                    # tokens of any magnitude
        wide = wide.to(DTYPE[case["dtype"]])
        s["k"], s["v"] = wide[:, :case["kv_heads"]], wide[:, case["kv_heads"]:]
    else:
        s["q"] = wide.to(torch.bfloat16)[:, :heads]
    return s


# ------------------------------------------------------------------------------- one pass
def _plain_codes(s):
    side, rows, cols = s["side"], s["rows"], s["cols"]
    full = torch.zeros(_up(rows, side), _up(cols, SIDE), device="cuda")
    full[:rows, :cols] = s["x"].float()
    tiles = full.view(full.shape[0] // side, side, full.shape[1] // SIDE, SIDE)
    top = tiles.abs().amax((1, 3))
    delta = torch.where(top > 0, top / s["qmax"], torch.ones_like(top))
    t = (tiles / delta[:, None, :, None]).clamp(-QMAX[s["fmt"]], QMAX[s["fmt"]])
    return {"codes": t.view(full.shape)[:rows, :cols].to(HELD[s["fmt"]]), "delta": delta.t().contiguous()}


def _wide_matrix(codes, delta, fmt, k, side):
    rows = codes.shape[0]
    scales = delta.t().repeat_interleave(side, 0)[:rows].repeat_interleave(SIDE, 1)[:, :k]
    return codes.view(HELD[fmt])[:, :k].float() * scales


def _plain_product(s):
    y = _wide_matrix(s["cx"], s["dx"], s["fmt_x"], s["k"], 1) @ _wide_matrix(s["cw"], s["dw"], s["fmt_w"], s["k"], s["side"]).t()
    return (y if s["b"] is None else y + s["b"]).to(DTYPE[s["out"]])


def _places(s, tokens):
    """Of each new token: its sequence, its number there among the new ones, and its position."""
    lens, starts = s["lens"].long(), s["starts"]
    starts = torch.arange(len(lens) + 1, device="cuda") if starts is None else starts.long()
    t = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(starts, t, right=True) - 1
    return seq, t - starts[seq], lens[seq] - starts[seq + 1] + t


def _requantize(values, delta, fmt):
    # codes of fp32 values under scales that may be 0, where every value is
    t = torch.where(delta > 0, values / delta, torch.zeros_like(values)).clamp(-QMAX[fmt], QMAX[fmt])
    return (t.round() if fmt == "int8" else t).to(HELD[fmt])


def _plain_append(s):
    # a block's scale covers the largest magnitude that it has held: where new tokens raise it, older codes are rounded again
    fmt, block = s["fmt"], s["block"]
    seq, number, pos = _places(s, s["k"].shape[0])
    page, slot = s["tables"][seq, pos // block].long(), pos % block
    begins = torch.nonzero((slot == 0) | (number == 0))[:, 0]          # the first new token of each block
    pages, held = page[begins], slot[begins]
    qmax = torch.tensor(QMAX[fmt], device="cuda")
    out = {}
    for name, x, codes, delta in (("k", s["k"], s["kc"], s["dk"]), ("v", s["v"], s["vc"], s["dv"])):
        x, stored = x.float(), codes.view(HELD[fmt])
        before = torch.where(held[:, None] > 0, delta[pages], torch.zeros_like(delta[pages]))
        top = torch.zeros_like(delta).index_reduce_(0, page, x.abs().amax(2), "amax")[pages]
        after = torch.maximum(before, top / qmax)
        old = stored[pages]
        again = _requantize(old.float() * before[:, :, None, None], after[:, :, None, None], fmt)
        changes = (after > before)[:, :, None, None] & (torch.arange(block, device="cuda")[:, None] < held[:, None, None, None])
        codes[pages] = torch.where(changes, again.view(torch.uint8), old.view(torch.uint8))
        delta[pages] = after
        codes[page, :, slot] = _requantize(x, delta[page][:, :, None], fmt).view(torch.uint8)
        out[name], out["delta_" + name] = stored, delta
    return out


def _plain_attention(s):
    fmt, block, kv, dim = s["fmt"], s["block"], s["kv_heads"], s["dim"]
    q, lens = s["q"], s["lens"].long()
    batch, tokens, group = len(lens), q.shape[0], s["heads"] // kv
    seq, number, pos = _places(s, tokens)
    pages = s["tables"][:, :(s["longest"] + block - 1) // block].long()

    def wide(codes, delta):
        x = codes.view(torch.int8)[pages].view(HELD[fmt]).float() * delta[pages][..., None, None]           # [batch, blocks, kv, block, dim]
        return x.transpose(1, 2).reshape(batch, kv, -1, dim)
    k, v = wide(s["kc"], s["dk"]), wide(s["vc"], s["dv"])
    rows = torch.zeros(batch, s["most_new"], kv, group, dim, device="cuda")
    rows[seq, number] = q.float().view(tokens, kv, group, dim)
    rows = rows.permute(0, 2, 1, 3, 4).reshape(batch, kv, -1, dim)
    scores = (rows @ k.transpose(2, 3) * dim ** -0.5).view(batch, kv, s["most_new"], group, -1)
    last = torch.full((batch, s["most_new"]), -1, device="cuda")
    last[seq, number] = pos                                            # a token sees itself and what is before it
    hidden = torch.arange(k.shape[2], device="cuda") > last[:, None, :, None, None]
    scores = scores.masked_fill_(hidden, float("-inf"))
    top = scores.amax(4, keepdim=True).clamp_min(-3e38)
    p = (scores - top).exp_()
    total = p.sum(4, keepdim=True)
    o = (p.view(batch, kv, -1, k.shape[2]) @ v).view(batch, kv, s["most_new"], group, dim) / total
    lse = (top + total.log())[..., 0]
    o, lse = o.permute(0, 2, 1, 3, 4)[seq, number], lse.permute(0, 2, 1, 3)[seq, number]
    return {"out": o.reshape(tokens, s["heads"], dim).to(torch.bfloat16), "lse": lse.reshape(tokens, s["heads"])}


def run(s):
    if own:
        import paper_2408_02897_b200 as qm
        if s["op"] == "codes":
            codes, delta = qm.qm_quantize_blocks(qm.operand_of(s["x"], -1), s["fmt"], side=s["side"])
            return {"codes": codes.view(HELD[s["fmt"]])[:, :s["cols"]], "delta": delta}
        if s["op"] == "product":
            return qm.qm_linear_fp8(s["cx"], s["dx"], s["cw"], s["dw"], s["k"], s["fmt_x"], s["fmt_w"], side_w=s["side"], bias=s["b"],
                                    out_dtype=DTYPE[s["out"]])
        if s["op"] == "append":
            qm.qm_cache_append(s["k"], s["v"], s["kc"], s["dk"], s["vc"], s["dv"], s["tables"], s["lens"], s["starts"], fmt=s["fmt"])
            return {"k": s["kc"].view(HELD[s["fmt"]]), "delta_k": s["dk"], "v": s["vc"].view(HELD[s["fmt"]]), "delta_v": s["dv"]}
        out, lse = qm.qm_cache_attention(s["q"], s["kc"], s["dk"], s["vc"], s["dv"], s["tables"], s["lens"], s["starts"], fmt=s["fmt"],
                                         want_lse=True)
        return {"out": out, "lse": lse}
    return {"codes": _plain_codes, "product": _plain_product, "append": _plain_append, "attention": _plain_attention}[s["op"]](s)


# ------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Of ragged batches, what their lengths come to on the average: uniform from 1 to the largest, one of them being that."""
    if case["op"] == "codes":
        n, scales = case["rows"] * case["cols"], (case["rows"] + case["side"] - 1) // case["side"] * ((case["cols"] + SIDE - 1) // SIDE)
        return {"bytes": n * (3 if case["dtype"] == "bf16" else 5) + 4 * scales, "flops": 3 * n}
    if case["op"] == "product":
        m, n, k, es = case["m"], case["n"], case["k"], 2 if case["out"] == "bf16" else 4
        scales = (k + SIDE - 1) // SIDE * (m + (n + case["side"] - 1) // case["side"])
        return {"bytes": m * k + n * k + 4 * scales + m * n * es + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}

    def total(most):
        return case["batch"] * most if case.get("even") else int((case["batch"] - 1) * (1 + most) / 2 + most)
    tokens, row = total(case["most_new"]), case["kv_heads"] * case["dim"]
    if case["op"] == "append":
        blocks = tokens // case["block"] + case["batch"]
        return {"bytes": 2 * tokens * row * ((2 if case["dtype"] == "bf16" else 4) + 1) + 8 * blocks * case["kv_heads"], "flops": 6 * tokens * row}
    kept = total(case["most_len"])
    seen = kept / case["batch"] - (tokens / case["batch"] - 1) / 2      # keys of a query, about
    blocks = kept // case["block"] + case["batch"]
    return {"bytes": 2 * kept * row + 8 * blocks * case["kv_heads"] + 4 * blocks + tokens * case["heads"] * (4 * case["dim"] + 4),
            "flops": int(4 * tokens * seen * case["heads"] * case["dim"])}


# ------------------------------------------------------------------------------- the definition, in 64 bits
def _nearest(t, fmt):
    """The nearest value of the format's grid, ties to the even code; t is within its range."""
    if fmt == "int8":
        return torch.round(t)
    mantissa, least = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(t.abs().clamp_min(2.0 ** least))[1] - 1            # 2^e <= |t|, at least the smallest normal's
    step = torch.ldexp(torch.ones_like(t), e - mantissa)
    return torch.round(t / step) * step


def _exact_codes(case, s):
    x, side = s["x"].double(), case["side"]
    codes, delta = torch.empty_like(x), []
    for c in range(0, case["cols"], SIDE):
        part = x[:, c:c + SIDE]
        top = torch.stack([p.abs().max() for p in part.split(side)]) if side > 1 else part.abs().max(1).values
        d = torch.where(top > 0, top / QMAX[case["fmt"]], torch.ones_like(top))
        codes[:, c:c + SIDE] = _nearest(part / d.repeat_interleave(side)[:case["rows"], None], case["fmt"])
        delta.append(d)
    return {"codes": codes, "delta": torch.stack(delta)}


def _exact_append(case, s):
    fmt, block, out = case["fmt"], case["block"], {}
    lens = s["lens"].tolist()
    starts = list(range(len(lens) + 1)) if s["starts"] is None else s["starts"].tolist()
    tables = s["tables"].tolist()
    for name, x, codes, delta in (("k", s["k"], s["kc"], s["dk"]), ("v", s["v"], s["vc"], s["dv"])):
        values, scales = codes.view(HELD[fmt]).double(), delta.double()
        for b, length in enumerate(lens):
            fresh, pos = x[starts[b]:starts[b + 1]].double().transpose(0, 1), length - (starts[b + 1] - starts[b])     # [heads, new, dim]
            while pos < length:
                page, first = tables[b][pos // block], pos % block
                n = min(block - first, length - pos)
                part = fresh[:, :n]
                fresh = fresh[:, n:]
                pos += n
                old = values[page, :, :first] * scales[page][:, None, None]
                both = torch.cat([old, part], 1)
                d = part.abs().amax((1, 2)) / QMAX[fmt]
                if first:
                    grows = d > scales[page]
                    d = torch.maximum(d, scales[page])
                    again = _nearest(both[:, :first] / d[:, None, None], fmt)
                    values[page, :, :first] = torch.where(grows[:, None, None], again, values[page, :, :first])
                values[page, :, first:first + n] = _nearest(part / d[:, None, None], fmt)
                scales[page] = d
        out[name], out["delta_" + name] = values.to(torch.int8) if fmt == "int8" else values, scales
    return out


def _exact_attention(case, s):
    fmt, block, heads, kv = case["fmt"], case["block"], case["heads"], case["kv_heads"]
    lens = s["lens"].tolist()
    starts = list(range(len(lens) + 1)) if s["starts"] is None else s["starts"].tolist()
    outs, logs = [], []
    for b, length in enumerate(lens):
        n = starts[b + 1] - starts[b]
        pages = s["tables"][b, :(length + block - 1) // block].long()
        k, v = ((c.view(torch.int8)[pages].view(HELD[fmt]).double() * d[pages].double()[:, :, None, None]).permute(1, 0, 2, 3).flatten(1, 2)[:, :length]
                for c, d in ((s["kc"], s["dk"]), (s["vc"], s["dv"])))
        q = s["q"][starts[b]:starts[b + 1]].double().view(n, kv, heads // kv, case["dim"])
        o, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float64, device="cuda")
        for h in range(kv):
            scores = torch.einsum("ngd,kd->ngk", q[:, h], k[h]) / math.sqrt(case["dim"])
            later = torch.arange(length, device="cuda")[None, :] > length - n + torch.arange(n, device="cuda")[:, None]
            scores.masked_fill_(later[:, None, :], float("-inf"))
            lse[:, h] = torch.logsumexp(scores, 2)
            o[:, h] = torch.einsum("ngk,kd->ngd", torch.softmax(scores, 2), v[h])
        outs.append(o.reshape(n, heads, -1))
        logs.append(lse.reshape(n, heads))
    return {"out": torch.cat(outs), "lse": torch.cat(logs)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "codes":
        return _exact_codes(case, s)
    if case["op"] == "append":
        return _exact_append(case, s)
    if case["op"] == "attention":
        return _exact_attention(case, s)
    y = torch.zeros(case["m"], case["n"], dtype=torch.float64, device="cuda")
    for c in range(0, case["k"], SIDE):
        a = s["cx"].view(HELD[case["fmt_x"]])[:, c:min(c + SIDE, case["k"])].double() * s["dx"][c // SIDE].double()[:, None]
        w = s["cw"].view(HELD[case["fmt_w"]])[:, c:min(c + SIDE, case["k"])].double()
        y += a @ (w * s["dw"][c // SIDE].double().repeat_interleave(case["side"])[:case["n"], None]).t()
    return y if s["b"] is None else y + s["b"].double()
