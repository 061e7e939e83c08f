"""The operators that serve many requests at once from decoded weights, as measured work.

Four operators, in the order in which a step of a serving program calls them:

* ``tables``:   block tables, slot maps and row ranges of a batch, made on the GPU from the requests' lengths;
* ``adapters``: each request's low-rank adapter beside a projection that all requests share;
* ``write``:    keys and values into a paged cache of 8-bit codes with one scale for each block (page) and head;
* ``attend``:   attention of the new tokens over that cache, for prompts, chunks and single tokens.

``own = False`` computes them by elementary torch operations in 32 bits; ``own = True`` makes the
framework's calls on the same state.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -40                                # of a block of the cache


def listed():
    return [
        # a decode step of 64 sequences: one token each, few of them start a page
        dict(name="tables step", op="tables", seqs=64, new=1, context=1500, page=16, room=0),
        # many requests admitted at once, ragged prompts, rows padded to a captured graph's size
        dict(name="tables prompts", op="tables", seqs=700, new=301, context=4001, page=16, room=1000),
        # one row of a narrow model through one adapter: latency
        dict(name="adapters token", op="adapters", seqs=1, new=1, x="bf16", n_in=1024, n_out=1000, rank=8, count=4),
        # a decode step of 64 requests with an adapter each, beside the large dense layer (8192 x 8192)
        dict(name="adapters step", op="adapters", seqs=64, new=1, x="bf16", n_in=8192, n_out=8192, rank=16, count=100),
        # ragged prompts of a few requests, their rows in 8 bits from the norm
        dict(name="adapters prompts 8-bit", op="adapters", seqs=7, new=1001, x="e4m3", n_in=8192, n_out=8192, rank=32, count=16),
        # one new token of one short sequence: latency
        dict(name="write token", op="write", seqs=1, new=1, context=100, heads=8, dim=128, page=16, x="bf16"),
        # chunks of new tokens behind cached ones
        dict(name="write chunk", op="write", seqs=5, new=2048, context=6001, heads=8, dim=128, page=64, x="bf16"),
        # one token of one short sequence: latency
        dict(name="attend token", op="attend", seqs=1, new=1, context=100, heads=8, share=4, dim=128, page=16, window=0, causal=True),
        # a decode step of 64 sequences
        dict(name="attend step", op="attend", seqs=64, new=1, context=1500, heads=8, share=4, dim=128, page=16, window=0, causal=True),
        # one token of one long sequence, eight queries a head of the cache
        dict(name="attend long", op="attend", seqs=1, new=1, context=32768, heads=8, share=8, dim=128, page=64, window=0, causal=True),
        # a whole prompt
        dict(name="attend prompt", op="attend", seqs=1, new=4096, context=0, heads=8, share=4, dim=128, page=64, window=0, causal=True),
        # chunks of prompts behind cached tokens, ragged
        dict(name="attend chunk", op="attend", seqs=5, new=2048, context=6001, heads=8, share=4, dim=128, page=64, window=0, causal=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "adapters", "write", "attend", "attend"))
    if op == "tables":
        seqs = _log(rng, 1, 2000)
        new = 1 if rng.random() < 0.4 else _log(rng, 1, max(1, min(8000, 200000 // seqs)))
        return dict(op=op, seqs=seqs, new=new, context=_log(rng, 1, min(16000, 8000000 // seqs)), page=rng.choice((16, 32, 48, 64, 128)),
                    room=rng.choice((0, 0, 7, 500)))
    if op == "adapters":
        n_in, n_out = _log(rng, 64, 8192), _log(rng, 64, 8192)
        if rng.random() < 0.8:
            n_in, n_out = (n_in + 15) // 16 * 16, (n_out + 15) // 16 * 16
        seqs = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.5 else _log(rng, 1, 7000 // seqs)
        return dict(op=op, seqs=seqs, new=new, x=rng.choice(("bf16", "bf16", "e4m3")), n_in=n_in, n_out=n_out,
                    rank=rng.choice((4, 8, 16, 16, 32, 64)), count=rng.choice((1, 8, 64)))
    dim, page, heads = rng.choice((64, 80, 128, 128, 256)), rng.choice((16, 32, 48, 64, 128)), rng.choice((1, 2, 4, 8))
    seqs = _log(rng, 1, 64)
    if op == "write":
        new = 1 if rng.random() < 0.4 else _log(rng, 1, max(1, 10240 * 1024 // (heads * dim * seqs)))
        return dict(op=op, seqs=seqs, new=min(new, 4096), context=_log(rng, 1, 8000), heads=heads, dim=dim, page=page, x=rng.choice(("bf16", "bf16", "f32")))
    share = rng.choice((1, 2, 4, 4, 7, 8))
    most = 64 * 1500 * 8 * 128 // (seqs * heads * dim)               # cached tokens a sequence may have
    context = min(_log(rng, 16, 32768), most)
    pairs = 5 * 2048 * 7000 * 32 * 128 // (seqs * heads * share * dim)  # of a new token and a cached one
    new = 1
    if rng.random() < 0.6:
        new = _log(rng, 2, 4096)
        new = max(1, min(new, pairs // max(context, 1), math.isqrt(pairs)))
    return dict(op=op, seqs=seqs, new=new, context=context, heads=heads, share=share, dim=dim, page=page,
                window=rng.choice((0, 0, 0, 100, 1024)), causal=True if new == 1 else rng.random() < 0.8)


# ---- inputs --------------------------------------------------------------------------------------
def _ragged(n, most, least):
    """Numbers between about a half and the whole of `most`."""
    return [max(least, most - (most * i * 5 // (n * 10))) for i in range(n)]


def _lengths(case):
    """(tokens cached before the call, new tokens) of each sequence."""
    n = case["seqs"]
    return _ragged(n, case["context"], 0), _ragged(n, case["new"], 1)[::-1]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    return torch.nn.functional.pad(_int32(counts).cumsum(0), (1, 0)).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    s = {"case": case, "op": case["op"]}
    if case["op"] == "adapters":
        new = _ragged(case["seqs"], case["new"], 1)
        rows, n_in, n_out, rank, count = sum(new), case["n_in"], case["n_out"], case["rank"], case["count"]
        s["new"], s["starts"], s["rows"] = new, _starts(new), rows
        x = normal(rows, n_in)
        s["x_scales"] = None
        if case["x"] == "e4m3":
            s["x_scales"] = x.abs().amax(1) / E4M3_MAX
            x = x / s["x_scales"][:, None]
        s["x"] = x.to(E4M3 if case["x"] == "e4m3" else torch.bfloat16)
        s["a"] = (normal(count, rank, n_in) / math.sqrt(n_in)).to(torch.bfloat16)
        s["b"] = (0.3 * normal(count, n_out, rank) / math.sqrt(rank)).to(torch.bfloat16)
        s["scales"] = 0.5 + torch.rand(count, device="cuda", generator=gen)
        s["which"] = torch.randperm(max(count, case["seqs"]), device="cuda", generator=gen)[:case["seqs"]].remainder(count).to(torch.int32)
        if case["seqs"] > 4:
            s["which"][3] = -1                                         # a request without an adapter
        s["y"] = normal(rows, n_out).to(torch.bfloat16)                # of the shared projection
        s["out"] = torch.empty_like(s["y"])
    else:
        before, new = _lengths(case)
        page, n = case["page"], case["seqs"]
        after = [b + m for b, m in zip(before, new)]
        held, need = ([-(-c // page) for c in t] for t in (before, after))
        s["cached"], s["new"], s["lengths"], s["starts"] = _int32(before), _int32(new), _int32(after), _starts(new)
        s["rows"], s["most_new"], s["most"] = sum(new), max(new), max(after)
        n_pages = sum(need) + 5
        order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
        pages = max(need) + 2
        place = torch.arange(pages, device="cuda")
        rank = _starts(need)[:-1, None] + place                        # pages of a sequence lie anywhere
        if case["op"] == "tables":
            s["free"], s["taken"] = order, _int32([sum(held)])
            rank = _starts(held)[:-1, None] + place
            s["tables"] = torch.where(place < _int32(held)[:, None], order[rank.clamp(max=n_pages - 1)], -1)
            s["room"] = s["rows"] + case["room"]
        else:
            heads, dim = case["heads"], case["dim"]
            s["tables"] = torch.where(place < _int32(need)[:, None], order[rank.clamp(max=n_pages - 1)], 0)
            for t in "kv":                                             # what earlier calls have written
                codes = (40 * torch.randn(n_pages, heads, page, dim, device="cuda", generator=gen)).round_().clamp_(-127, 127)
                s[t + "_codes"] = codes.to(torch.int8)
                s[t + "_scales"] = torch.exp2(torch.randint(-6, -4, (n_pages, heads), device="cuda", generator=gen).float())
            if case["op"] == "write":                                  # the products' output holds queries, keys and values side by side
                dt = torch.float32 if case["x"] == "f32" else torch.bfloat16
                qkv = (normal(s["rows"], 3, heads, dim) + 0.5 * normal(3, heads, dim)).to(dt)
                s["k"], s["v"] = qkv[:, 1], qkv[:, 2]
            else:
                s["q"] = (0.7 * normal(s["rows"], heads * case["share"], dim)).to(torch.bfloat16)
                s["out"] = torch.empty_like(s["q"])
    if own:                                                            # the handles and buffers that a program keeps; no data is touched
        from paper_2406_06237_b200 import runtime
        if s["op"] == "tables":
            s["handle"] = runtime.PageTables(case["page"])
            s["batch"] = s["handle"].buffers(case["seqs"], s["room"])
        elif s["op"] == "adapters":
            s["handle"] = runtime.Adapters(s["a"], s["b"], s["scales"])
        else:
            s["handle"] = runtime.BlockCache.wrap(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
    return s


# ---- one pass ------------------------------------------------------------------------------------
def _tables(s):
    page, cached, new, taken = s["case"]["page"], s["cached"], s["new"], s["taken"]
    lengths = cached + new
    starts, ends = (torch.nn.functional.pad(t.cumsum(0), (1, 0)).to(torch.int32) for t in (new, lengths))
    held, need = (cached + page - 1) // page, (lengths + page - 1) // page
    more = need - held
    first = taken + more.cumsum(0) - more                              # of a request's new pages, in the free list
    place = torch.arange(s["tables"].shape[1], device="cuda")
    fresh = (place >= held[:, None]) & (place < need[:, None])
    given = s["free"][torch.where(fresh, first[:, None] + place - held[:, None], 0)]
    s["tables"].copy_(torch.where(fresh, given, s["tables"]))
    rows = torch.arange(s["room"], device="cuda", dtype=torch.int32)
    live = rows < starts[-1]
    seq = (torch.searchsorted(starts, rows, right=True) - 1).clamp(max=new.shape[0] - 1)
    positions = torch.where(live, cached[seq] + rows - starts[seq], 0)
    slots = s["tables"][seq, positions // page].long() * page + positions % page
    return {"tables": s["tables"], "starts": starts, "lengths": lengths, "ends": ends, "slots": torch.where(live, slots, -1),
            "positions": positions, "taken": taken + more.sum().to(torch.int32)}


def _sequences(s):
    """Sequence of each row and its number within the sequence."""
    rows = torch.arange(s["rows"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], rows, right=True) - 1
    return seq, rows - s["starts"][seq]


def _adapters(s):
    seq, at = _sequences(s)
    x = s["x"].float()
    if s["x_scales"] is not None:
        x = x * s["x_scales"][:, None]
    which = s["which"].long()
    padded = torch.zeros(len(s["new"]), max(s["new"]), x.shape[1], device="cuda")
    padded[seq, at] = x
    h = padded @ s["a"][which].float().transpose(1, 2) * torch.where(which < 0, 0, s["scales"][which])[:, None, None]
    return (s["y"].float() + (h @ s["b"][which].float().transpose(1, 2))[seq, at]).to(s["y"].dtype)


def _power(top):
    """The least power of two that holds `top` in 127 steps."""
    m, e = torch.frexp(top)
    return torch.ldexp(torch.ones_like(top), e - 7 + (m > 127 / 128)).clamp(min=LEAST_SCALE)


def _write(s):
    page, n = s["case"]["page"], s["case"]["seqs"]
    cached, lengths = s["cached"].long(), s["lengths"].long()
    blocks = cached[:, None] // page + torch.arange((s["most_new"] + page - 2) // page + 1, device="cuda")   # those that get new tokens
    seq, block = torch.nonzero(blocks * page < lengths[:, None], as_tuple=True)
    block = blocks[seq, block]
    pages = s["tables"][seq, block].long()
    at = block[:, None] * page + torch.arange(page, device="cuda")     # positions of a block's tokens
    kept, fresh = at < cached[seq, None], (at >= cached[seq, None]) & (at < lengths[seq, None])
    row = torch.where(fresh, s["starts"][seq, None] + at - cached[seq, None], 0)
    for t in "kv":
        codes, scales = s[t + "_codes"], s[t + "_scales"]
        x = s[t][row].float().transpose(1, 2)                          # [block, head, token, dim]
        top = torch.where(fresh[:, None, :, None], x, 0).abs().amax((2, 3))
        old = scales[pages]
        scale = torch.where(kept.any(1)[:, None], torch.maximum(old, _power(top)), _power(top))
        old_codes = codes[pages]
        value = torch.where(kept[:, None, :, None], old_codes.float() * old[..., None, None], x)
        q = torch.round(value / scale[..., None, None]).to(torch.int8)
        codes[pages] = torch.where((kept | fresh)[:, None, :, None], q, old_codes)
        scales[pages] = scale
    return {f: s[f] for f in ("k_codes", "k_scales", "v_codes", "v_scales")}


def _attend(s):
    case = s["case"]
    n, heads, share, dim, most = case["seqs"], case["heads"], case["share"], case["dim"], s["most"]
    pages = s["tables"][:, :-(-most // case["page"])].long()
    k, v = ((s[t + "_codes"][pages].float() * s[t + "_scales"][pages][..., None, None]).transpose(2, 3).flatten(1, 2)[:, :most] for t in "kv")
    seq, at = _sequences(s)
    q = torch.zeros(n, s["most_new"], heads, share, dim, device="cuda")
    q[seq, at] = s["q"].unflatten(1, (heads, share)).float()
    q = q.permute(0, 2, 3, 1, 4).flatten(2, 3)                         # [sequence, head, query, dim]
    score = q @ k.permute(0, 2, 3, 1) * dim ** -0.5
    lengths = s["lengths"][:, None]
    end = lengths - (s["starts"][1:] - s["starts"][:-1])[:, None] + torch.arange(s["most_new"], device="cuda") + 1 if case["causal"] \
        else lengths.expand(n, s["most_new"])
    token = torch.arange(most, device="cuda")
    hidden = token >= end[..., None]
    if case["window"]:
        hidden = hidden | (token < end[..., None] - case["window"])
    score = score.unflatten(2, (share, -1)).masked_fill_(hidden[:, None, None], float("-inf")).flatten(2, 3)
    p = torch.exp(score.sub_(score.amax(3, keepdim=True).clamp(min=-3e38)))
    total = p.sum(3, keepdim=True)
    out = (p @ v.transpose(1, 2) / total.clamp(min=1e-38)).unflatten(2, (share, -1))
    return out.permute(0, 3, 1, 2, 4)[seq, at].flatten(1, 2).to(torch.bfloat16)


def run(s):
    if not own:
        return {"tables": _tables, "adapters": _adapters, "write": _write, "attend": _attend}[s["op"]](s)
    f, case = s["handle"], s["case"]
    if s["op"] == "tables":
        batch = f(s["tables"], s["cached"], s["new"], s["free"], s["taken"], out=s["batch"])
        return {"tables": s["tables"], **batch._asdict()}
    if s["op"] == "adapters":
        return f(s["x"], s["y"], s["which"], s["starts"], x_scales=s["x_scales"], out=s["out"])
    if s["op"] == "write":
        f.write(s["k"], s["v"], s["tables"], s["lengths"], s["starts"])
        return {t: s[t] for t in ("k_codes", "k_scales", "v_codes", "v_scales")}
    return f.attend(s["q"], s["tables"], s["lengths"], s["starts"], causal=case["causal"], window=case["window"], longest=s["most_new"], out=s["out"])


# ---- what a pass cannot do without ---------------------------------------------------------------
def _seen(case):
    """(pairs of a query token and a cached one that it sees, cached tokens that a query sees) over all sequences."""
    pairs = tokens = 0
    for b, m in zip(*_lengths(case)):
        w = case["window"] or b + m
        if case["causal"]:
            ends = range(b + 1, b + m + 1)
            pairs += sum(min(e, w) for e in ends)
            tokens += b + m - max(0, b + 1 - w)
        else:
            pairs += m * min(b + m, w)
            tokens += min(b + m, w)
    return pairs, tokens


def work(case):
    if case["op"] == "adapters":
        new = _ragged(case["seqs"], case["new"], 1)
        rows, r = sum(new), case["rank"]
        used = min(case["count"], case["seqs"])
        b = rows * (case["n_in"] * (1 if case["x"] == "e4m3" else 2) + 4 * case["n_out"]) + used * 2 * r * (case["n_in"] + case["n_out"])
        return {"bytes": b, "flops": 2 * rows * r * (case["n_in"] + case["n_out"])}
    before, new = _lengths(case)
    rows, page = sum(new), case["page"]
    held, need = (sum(-(-(b + m * k) // page) for b, m in zip(before, new)) for k in (0, 1))
    if case["op"] == "tables":
        last = case["seqs"] if case["new"] == 1 else 0                 # cached pages that are looked at: those that get tokens
        return {"bytes": 12 * (rows + case["room"]) + 20 * case["seqs"] + 8 * (need - held) + 4 * last, "flops": 0}
    heads, dim = case["heads"], case["dim"]
    if case["op"] == "write":
        part = sum(b % page for b in before if b % page)               # tokens whose block may get another scale
        touched = sum(-(-(b + m) // page) - b // page for b, m in zip(before, new))
        row = 2 * heads * dim
        return {"bytes": rows * row * ((4 if case["x"] == "f32" else 2) + 1) + touched * (2 * heads * 4 + 4), "flops": 3 * rows * row}
    pairs, tokens = _seen(case)
    b = 2 * tokens * heads * dim + 4 * rows * heads * case["share"] * dim + (tokens // page) * (4 + 8 * heads)
    return {"bytes": b, "flops": 4 * pairs * heads * case["share"] * dim}


# ---- the definition in 64 bits -------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"] == "tables":
        page, free, taken = case["page"], s["free"].tolist(), int(s["taken"])
        tables, slots, positions, starts, ends = s["tables"].tolist(), [], [], [0], [0]
        for i, (b, m) in enumerate(zip(s["cached"].tolist(), s["new"].tolist())):
            for j in range(-(-b // page), -(-(b + m) // page)):
                tables[i][j] = free[taken]
                taken += 1
            positions += range(b, b + m)
            slots += [tables[i][p // page] * page + p % page for p in range(b, b + m)]
            starts.append(starts[-1] + m)
            ends.append(ends[-1] + b + m)
        rest = s["room"] - len(slots)
        return {"tables": _int32(tables), "starts": _int32(starts), "lengths": s["lengths"], "ends": _int32(ends),
                "slots": torch.tensor(slots + [-1] * rest, device="cuda"), "positions": _int32(positions + [0] * rest), "taken": _int32([taken])}
    if case["op"] == "adapters":
        y = s["y"].to(d)
        at = 0
        for m, i in zip(s["new"], s["which"].tolist()):
            if i >= 0:
                x = s["x"][at:at + m].to(d)
                if s["x_scales"] is not None:
                    x = torch.einsum("ti,t->ti", x, s["x_scales"][at:at + m].to(d))
                y[at:at + m] += torch.einsum("ti,ri,or->to", x, s["a"][i].to(d), s["b"][i].to(d) * s["scales"][i].to(d))
            at += m
        return y
    page = case["page"]
    lists = zip(s["cached"].tolist(), s["lengths"].tolist(), s["starts"].tolist(), s["tables"])
    if case["op"] == "write":
        if sum(-(-m // page) + 1 for m in _lengths(case)[1]) > 3000:
            return None
        out = {t + f: s[t + f].to(d) for t in "kv" for f in ("_codes", "_scales")}
        for before, after, start, table in lists:
            for j in range(before // page, -(-after // page)):
                p, lo, hi = int(table[j]), max(before, j * page), min(after, (j + 1) * page)
                for t in "kv":
                    codes, scales = out[t + "_codes"][p], out[t + "_scales"][p]
                    x = s[t][start + lo - before:start + hi - before].to(d).transpose(0, 1)
                    step = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / 127))).clamp(min=LEAST_SCALE)
                    if lo > j * page:
                        step = torch.maximum(step, scales)
                        old = codes[:, :lo - j * page] * scales[:, None, None]
                        codes[:, :lo - j * page] = torch.round(old / step[:, None, None])
                    codes[:, lo - j * page:hi - j * page] = torch.round(x / step[:, None, None])
                    scales.copy_(step)
        return {f: t.to(torch.int8) if f.endswith("codes") else t for f, t in out.items()}
    heads, share, dim = case["heads"], case["share"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=d, device="cuda")
    for before, after, start, table in lists:
        pages = table[:-(-after // page)].long()
        k, v = ((s[t + "_codes"][pages].to(d) * s[t + "_scales"][pages].to(d)[:, :, None, None]).transpose(0, 1).flatten(1, 2)[:, :after] for t in "kv")
        m = after - before
        for lo in range(0, m, 512):
            hi = min(m, lo + 512)
            q = s["q"][start + lo:start + hi].to(d).unflatten(1, (heads, share))
            score = torch.einsum("thgd,hsd->hgts", q, k) / math.sqrt(dim)
            last = torch.arange(before + lo, before + hi, device="cuda")[:, None] if case["causal"] else torch.full((hi - lo, 1), after - 1, device="cuda")
            token = torch.arange(after, device="cuda")
            seen = token <= last
            if case["window"]:
                seen &= token > last - case["window"]
            p = torch.softmax(torch.where(seen, score, -math.inf), 3)
            out[start + lo:start + hi] = torch.einsum("hgts,hsd->thgd", p, v).flatten(1, 2)
    return out
