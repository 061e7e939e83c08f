"""The operators around the weight products of a language model, as measured work.

Three operators that a program needs next to the decoder of compressed weights:

* ``norm``:    root-mean-square norm of a row with the residual's addition, its output in bf16 or
               in 8 bits (e4m3) with one scale a row;
* ``product``: matrix product with the decoded weights, Y = act(X W^T + bias) + residual, with both
               operands in bf16 or both in 8 bits (e4m3) with scales of X's rows and W's rows;
* ``cache``:   keys and values quantised (zero-point, 8 or 4 bits) as they are written into a paged
               cache, and the sequences' keys and values read back out of it.

``own = False`` computes them by elementary torch operations in 32 bits; ``own = True`` makes the
framework's calls on the same state.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
TINY = torch.finfo(torch.float32).tiny
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": E4M3}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
EPS = 1e-6
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # one token of a decode step: the latency of the norm before a product with 8-bit rows
        dict(name="norm token", op="norm", rows=1, width=8192, x="bf16", out="e4m3", residual=True),
        # a prompt's rows of a wide model, with the residual stream carried in bf16
        dict(name="norm prompt", op="norm", rows=16384, width=8192, x="bf16", out="e4m3", residual=True),
        # a ragged batch whose width is no multiple of a vector of 8: rows start unaligned
        dict(name="norm odd width", op="norm", rows=1537, width=2047, x="bf16", out="bf16", residual=True),
        # the first norm of a model: no residual yet, rows from an embedding kept in 32 bits
        dict(name="norm f32", op="norm", rows=8192, width=4096, x="f32", out="bf16", residual=False),
        # one token against a large dense layer (8192 x 8192, the large-layer workload): weights in bf16
        dict(name="product token", op="product", m=1, n=8192, k=8192, x="bf16", act="silu", bias=True, residual=False),
        # a small decode batch against the same layer held in 8 bits, joined to the residual stream
        dict(name="product batch 8-bit", op="product", m=16, n=8192, k=8192, x="e4m3", act="none", bias=True, residual=True),
        # a classifier's product (2048 -> 1000) for a ragged batch
        dict(name="product ragged", op="product", m=333, n=1000, k=2048, x="bf16", act="gelu", bias=True, residual=False),
        # a prompt through the large dense layer, in bf16
        dict(name="product prompt", op="product", m=8192, n=8192, k=8192, x="bf16", act="gelu_tanh", bias=True, residual=False),
        # a prompt through the large dense layer, in 8 bits, joined to the residual stream
        dict(name="product prompt 8-bit", op="product", m=4096, n=8192, k=8192, x="e4m3", act="none", bias=False, residual=True),
        # one new token of one short sequence: latency
        dict(name="cache token", op="cache", seqs=1, new=1, context=100, heads=8, dim=128, page=16, bits=8, group=128),
        # a decode step of 64 sequences: one token each is written, all their contexts are read
        dict(name="cache step", op="cache", seqs=64, new=1, context=1500, heads=8, dim=128, page=16, bits=8, group=128),
        # chunks of new tokens behind cached ones, 4 bits with a scale for each 32 values
        dict(name="cache chunk 4-bit", op="cache", seqs=5, new=2048, context=6001, heads=8, dim=128, page=64, bits=4, group=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "product", "cache"))
    if op == "norm":
        rows, width = _log(rng, 1, 16384), _log(rng, 64, 16384)
        if rng.random() < 0.6:
            width = (width + 15) // 16 * 16
        rows = max(1, min(rows, 16384 * 8192 // width))
        return dict(op=op, rows=rows, width=width, x=rng.choice(("bf16", "bf16", "f32")),
                    out=rng.choice(("e4m3", "bf16")), residual=rng.random() < 0.6)
    if op == "product":
        k = _log(rng, 64, 8192)
        if rng.random() < 0.8:
            k = (k + 15) // 16 * 16
        return dict(op=op, m=_log(rng, 1, 8192), n=_log(rng, 64, 8192), k=k, x=rng.choice(("bf16", "e4m3")),
                    act=rng.choice(ACTIVATIONS), bias=rng.random() < 0.6, residual=rng.random() < 0.5)
    bits, dim = rng.choice((8, 4)), rng.choice((64, 80, 128, 256))
    group = rng.choice((dim, dim, 16 if dim == 80 else 32))
    heads, seqs = rng.choice((1, 2, 4, 8)), _log(rng, 1, 64)
    most = 96000 * 1024 // (heads * dim * seqs)              # tokens a sequence may have
    new = min(_log(rng, 1, 4096), most) if rng.random() < 0.5 else 1
    context = max(0, min(_log(rng, 16, 32768), most) - new)
    return dict(op=op, seqs=seqs, new=new, context=context, heads=heads, dim=dim, page=rng.choice((16, 32, 64, 48)),
                bits=bits, group=group)


# ---- inputs --------------------------------------------------------------------------------------
def _lengths(case):
    """Cached tokens of each sequence before the call: between a half and the whole of `context`."""
    n, c = case["seqs"], case["context"]
    return [c - (c * i * 5 // (n * 10)) for i in range(n)] if n > 1 else [c]


def _symbols(shape, bits, gen):
    """Zero-point quantised weights: Laplacian symbols around the zero-point, as integers q - zero."""
    u = torch.rand(shape, device="cuda", generator=gen) - 0.5
    lap = -torch.sign(u) * torch.log1p(-2 * u.abs().clamp(max=0.4999999))
    half = 1 << (bits - 1)
    return (lap * (half / 6)).round_().clamp_(-half, half - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    s = {"case": case, "op": case["op"]}
    if case["op"] == "norm":
        rows, width, dt = case["rows"], case["width"], DTYPES[case["x"]]
        spread = torch.exp(0.5 * normal(width))                        # some channels are larger than others
        s["x"] = (normal(rows, width) * spread).to(dt)
        s["residual"] = (2 * normal(rows, width) * spread).to(dt) if case["residual"] else None
        s["weight"] = (1 + 0.2 * normal(width)).to(torch.bfloat16)
        s["out"] = torch.empty(rows, width, dtype=DTYPES[case["out"]], device="cuda")
        s["scales"] = torch.empty(rows, device="cuda") if case["out"] == "e4m3" else None
        s["summed"] = torch.empty_like(s["x"]) if case["residual"] else None
    elif case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        x = normal(m, k)
        if case["x"] == "e4m3":
            s["x_scales"] = x.abs().amax(1).clamp(min=TINY) / E4M3_MAX
            s["x"] = (x / s["x_scales"][:, None]).to(E4M3)
            s["w"] = _symbols((n, k), 4, gen).to(E4M3)                 # q - zero of 4-bit weights: exact in e4m3
            s["w_scales"] = (0.5 + torch.rand(n, device="cuda", generator=gen)) / math.sqrt(2 * k)
        else:
            s["x"], s["x_scales"], s["w_scales"] = x.to(torch.bfloat16), None, None
            s["w"] = (_symbols((n, k), 8, gen) * (0.03 / math.sqrt(k))).to(torch.bfloat16)
        s["bias"] = 0.5 * normal(n) if case["bias"] else None
        s["residual"] = normal(m, n).to(torch.bfloat16) if case["residual"] else None
        s["out"] = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    else:
        heads, dim, page, bits, group = (case[f] for f in ("heads", "dim", "page", "bits", "group"))
        before = _lengths(case)
        after = [c + case["new"] for c in before]
        need = [-(-c // page) for c in after]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
        tables = torch.zeros(len(need), max(need), dtype=torch.int32, device="cuda")
        at = 0
        for i, c in enumerate(need):                                   # pages of a sequence lie anywhere
            tables[i, :c] = order[at:at + c]
            at += c
        old = torch.tensor(before, device="cuda")
        pos = (old[:, None] + torch.arange(case["new"], device="cuda")).reshape(-1)
        seq = torch.arange(len(before), device="cuda").repeat_interleave(case["new"])
        s["slots"] = tables[seq, pos // page].to(torch.int64) * page + pos % page
        s["tables"] = tables
        s["starts"] = torch.tensor([0] + after, device="cuda").cumsum(0).to(torch.int32)
        s["total"] = sum(after)
        # the products' output holds queries, keys and values side by side: rows of k and v are strided
        tokens = len(before) * case["new"]
        qkv = (normal(tokens, 3, heads, dim) + 0.5 * normal(3, heads, dim)).to(torch.bfloat16)
        s["k"], s["v"] = qkv[:, 1], qkv[:, 2]
        for t in "kv":                                                 # what earlier calls have written
            s[t + "_codes"] = torch.randint(0, 256, (n_pages, page, heads, dim * bits // 8), dtype=torch.uint8, device="cuda", generator=gen)
            s[t + "_scales"] = (4 + torch.rand(n_pages, page, heads, dim // group, device="cuda", generator=gen)) / (1 << bits)
            s[t + "_zeros"] = torch.randint((3 << bits) // 8, (5 << bits) // 8, (n_pages, page, heads, dim // group), dtype=torch.uint8, device="cuda", generator=gen)
            s[t + "_out"] = torch.empty(s["total"], heads, dim, dtype=torch.bfloat16, device="cuda")
    if own:                                                            # the handles that a program keeps; no data is touched
        from paper_2406_06237_b200 import runtime
        if s["op"] == "norm":
            s["handle"] = runtime.RmsNorm(s["weight"], EPS, out_dtype=s["out"].dtype)
        elif s["op"] == "product":
            s["handle"] = runtime.Linear(s["w"], scales=s["w_scales"], bias=s["bias"], activation=case["act"])
        else:
            s["handle"] = runtime.PagedCache.wrap(s["k_codes"], s["k_scales"], s["k_zeros"], s["v_codes"], s["v_scales"], s["v_zeros"], case["bits"])
    return s


# ---- one pass ------------------------------------------------------------------------------------
def _act(v, name):
    if name == "relu":
        return torch.clamp(v, min=0)
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def _norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    r = {"summed": h.to(s["x"].dtype)} if s["residual"] is not None else {}
    if s["scales"] is None:
        return {"out": y.to(s["out"].dtype), **r}
    scales = (y.abs().amax(1) / E4M3_MAX).clamp(min=TINY)
    return {"out": (y / scales[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3), "scales": scales, **r}


def _product(s):
    y = s["x"].float() @ s["w"].float().T
    if s["x_scales"] is not None:
        y = y * s["x_scales"][:, None] * s["w_scales"]
    if s["bias"] is not None:
        y = y + s["bias"]
    y = _act(y, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["out"].dtype)


def _quantise(x, bits, group):
    """Codes, scales and zero-points of rows [tokens, heads, dim] in groups; zero is always representable."""
    levels = (1 << bits) - 1
    x = x.float().unflatten(2, (-1, group))
    lo, hi = x.amin(3).clamp(max=0), x.amax(3).clamp(min=0)
    scale = (hi / levels - lo / levels).clamp(min=TINY)
    zero = torch.round(-lo / scale).clamp(0, levels)
    q = (torch.round(x / scale[..., None]) + zero[..., None]).clamp(0, levels)
    return q.flatten(2), scale, zero


def _cache(s):
    case, out = s["case"], []
    bits, group, page = case["bits"], case["group"], case["page"]
    rows = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], rows, right=True) - 1
    pos = rows - s["starts"][seq]
    slots = s["tables"][seq, pos // page].long() * page + pos % page
    for t in "kv":
        codes, scales, zeros = (s[t + f].flatten(0, 1) for f in ("_codes", "_scales", "_zeros"))
        q, scale, zero = _quantise(s[t], bits, group)
        q = q.to(torch.uint8)
        codes[s["slots"]] = q if bits == 8 else q[..., 0::2] | q[..., 1::2] << 4
        scales[s["slots"]] = scale
        zeros[s["slots"]] = zero.to(torch.uint8)
        q = codes[slots]
        if bits == 4:
            q = torch.stack((q & 15, q >> 4), 3).flatten(2)
        x = (q.unflatten(2, (-1, group)).float() - zeros[slots][..., None].float()) * scales[slots][..., None]
        out.append(x.flatten(2).to(torch.bfloat16))
    return out


def run(s):
    if not own:
        return {"norm": _norm, "product": _product, "cache": _cache}[s["op"]](s)
    f = s["handle"]
    if s["op"] == "norm":
        out, scales, summed = f(s["x"], s["residual"], out=s["out"], scales=s["scales"], summed=s["summed"])
        r = {"out": out, "scales": scales, "summed": summed}
        return {k: v for k, v in r.items() if v is not None}
    if s["op"] == "product":
        return f(s["x"], x_scales=s["x_scales"], residual=s["residual"], out=s["out"])
    f.write(s["k"], s["v"], s["slots"])
    return list(f.read(s["tables"], s["starts"], k_out=s["k_out"], v_out=s["v_out"]))


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        b = n * (SIZE[case["x"]] * (3 if case["residual"] else 1) + SIZE[case["out"]]) + 2 * case["width"]
        return {"bytes": b + (4 * case["rows"] if case["out"] == "e4m3" else 0), "flops": 6 * n}
    if case["op"] == "product":
        m, n, k, e = case["m"], case["n"], case["k"], SIZE[case["x"]]
        b = (m * k + n * k) * e + m * n * (4 if case["residual"] else 2) + (4 * n if case["bias"] else 0)
        return {"bytes": b + (4 * (m + n) if e == 1 else 0), "flops": 2 * m * n * k}
    tokens, total = case["seqs"] * case["new"], sum(_lengths(case)) + case["seqs"] * case["new"]
    row = case["heads"] * case["dim"]
    held = row * case["bits"] // 8 + 5 * (row // case["group"])      # a token's codes, scales and zero-points
    b = 2 * (tokens * (2 * row + held) + total * (2 * row + held)) + 8 * tokens + 4 * (total // case["page"])
    return {"bytes": b, "flops": 2 * row * (6 * tokens + 2 * total)}


# ---- the definition in 64 bits -------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"] == "norm":
        h = s["x"].to(d) + (s["residual"].to(d) if case["residual"] else 0)
        rms = torch.sqrt(h.square().sum(1) / case["width"] + EPS)
        y = torch.einsum("ij,j,i->ij", h, s["weight"].to(d), 1 / rms)
        r = {"summed": h} if case["residual"] else {}
        if case["out"] != "e4m3":
            return {"out": y, **r}
        top = y.abs().max(1).values / E4M3_MAX
        return {"out": y / top[:, None], "scales": top, **r}
    if case["op"] == "product":
        y = torch.einsum("ik,jk->ij", s["x"].to(d), s["w"].to(d))
        if case["x"] == "e4m3":
            y = torch.einsum("ij,i,j->ij", y, s["x_scales"].to(d), s["w_scales"].to(d))
        if case["bias"]:
            y += s["bias"].to(d)
        if case["act"] == "relu":
            y = torch.where(y > 0, y, 0.0)
        elif case["act"] == "gelu":
            y = y * torch.special.ndtr(y)
        elif case["act"] == "gelu_tanh":
            y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        elif case["act"] == "silu":
            y = y / (1 + torch.exp(-y))
        return y + s["residual"].to(d) if case["residual"] else y
    levels, group, page = 2 ** case["bits"] - 1, case["group"], case["page"]
    starts, out = s["starts"].tolist(), []
    where = torch.cat([s["tables"][i].long().repeat_interleave(page)[:b - a] * page + torch.arange(b - a, device="cuda") % page
                       for i, (a, b) in enumerate(zip(starts, starts[1:]))])
    for t in "kv":
        q = s[t + "_codes"].flatten(0, 1)
        q = q if case["bits"] == 8 else torch.stack((q % 16, q // 16), -1).flatten(-2)
        held = q.to(d).unflatten(-1, (-1, group)) - s[t + "_zeros"].flatten(0, 1).to(d)[..., None]
        held = held * s[t + "_scales"].flatten(0, 1).to(d)[..., None]
        x = s[t].to(d).unflatten(-1, (-1, group))
        lo, hi = x.min(-1, keepdim=True).values.clamp(max=0), x.max(-1, keepdim=True).values.clamp(min=0)
        step = ((hi - lo) / levels).clamp(min=TINY)
        zero = torch.round(-lo / step)
        held[s["slots"]] = ((torch.round(x / step) + zero).clamp(0, levels) - zero) * step
        out.append(held.flatten(-2)[where])
    return out
