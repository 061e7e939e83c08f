"""What the tests of the operators on a batch of requests share: batches, and their definitions in 64 bits."""
import math

import torch

INT, BF16, F64 = torch.int32, torch.bfloat16, torch.float64
LEAST = 2.0 ** -40


def ints(values, device="cuda"):
    return torch.tensor(values, dtype=INT, device=device)


def sums(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def tables_for(lengths, page, seed=0, extra=3, wide=2):
    """Page tables for so many tokens each, pages anywhere, and the number of pages."""
    gen = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + extra
    order = torch.randperm(n_pages, generator=gen)
    tables = torch.full((len(lengths), max(need, default=0) + wide), -7, dtype=INT)
    for i, (at, n) in enumerate(zip(sums(need), need)):
        tables[i, :n] = order[at:at + n]
    return tables.cuda(), n_pages


def fill_cache(n_pages, heads, page, dim, seed=0, spread=3):
    """(codes, scales) twice: random codes, scales that are powers of two."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for _ in "kv":
        codes = (45 * torch.randn(n_pages, heads, page, dim, device="cuda", generator=gen)).round().clamp(-127, 127).to(torch.int8)
        out += [codes, torch.exp2(torch.randint(-6, spread - 6, (n_pages, heads), device="cuda", generator=gen).float())]
    return out


def values_of(codes, scales, table, length):
    """[heads, length, dim] in 64 bits."""
    page = codes.shape[2]
    pages = table[:-(-length // page)].long()
    return (codes[pages].to(F64) * scales[pages].to(F64)[:, :, None, None]).transpose(0, 1).flatten(1, 2)[:, :length]


def attention(q, arrays, tables, lengths, starts, scale=None, causal=True, window=0):
    """What attend() is: (result, the error that its arithmetic may have before the last rounding), in 64 bits.

    With p_i = exp(s_i) / sum: rounding p to fp16 is off by at most 2^-11 of it, so the result by 2^-11 sum p_i |v_i|.  A logit is
    a sum of up to 256 products in groups of 16 whose additions may each be off by 2^-22 of the sum of magnitudes B (17 of them),
    three roundings of factors follow and an exponential within 2^-22: under 2^-17 (1 + B) in all, which moves p_i and the sum
    of p by that share each.
    fp16 ends at steps of 2^-24: what is rounded is P_i = 2^u p_i c_i / T, u = 7 at least, c_i the scale of v_i's block and T the largest
    p_j c_j, so that a P_i under 2^-14 is off by up to 2^-25, half a step, and p_i v_i = P_i code_i T / 2^u by 2^-25 * 127 * T / 2^7:
    127 * 2^-32 T a token, which counts where the tokens with large p_i have a v_i of 0."""
    kc, ks, vc, vs = arrays
    heads, dim = kc.shape[1], kc.shape[3]
    share = q.shape[1] // heads
    scale = dim ** -0.5 if scale is None else scale
    out, slack = torch.zeros(q.shape, dtype=F64, device=q.device), torch.zeros(q.shape, dtype=F64, device=q.device)
    for s, length in enumerate(lengths):
        r0, r1 = starts[s], starts[s + 1]
        m = r1 - r0
        if m == 0 or length == 0:
            continue
        k, v = values_of(kc, ks, tables[s], length), values_of(vc, vs, tables[s], length)
        x = q[r0:r1].to(F64).unflatten(1, (heads, share))
        score = torch.einsum("thgd,hsd->hgts", x, k) * scale
        mass = torch.einsum("thgd,hsd->hgts", x.abs(), k.abs()) * abs(scale)
        token = torch.arange(length, device=q.device)
        last = torch.arange(length - m, length, device=q.device)[:, None] if causal else torch.full((m, 1), length - 1, device=q.device)
        seen = token <= last
        if window:
            seen &= token > last - window
        score = torch.where(seen, score, -math.inf)
        p = torch.where(seen, torch.exp(score - score.amax(3, keepdim=True).clamp(min=-1e300)), 0.0)
        total = p.sum(3, keepdim=True)
        p = torch.where(total > 0, p / total, 0.0)
        big = torch.where(seen, mass, 0.0).amax(3)                                     # B
        hidden = ~seen.any(1)                                                           # rows that see nothing are 0 whatever the values
        v0 = torch.where(p.sum(2).sum(1)[..., None] > 0, v, 0.0) if not torch.isfinite(v).all() else v
        at = torch.einsum("hgts,hsd->thgd", p, v0)
        at[hidden] = 0
        off = torch.einsum("hgts,hsd->thgd", p, v0.abs()) * (2.0 ** -11 + 2 * 2.0 ** -17 * (1 + big.permute(2, 0, 1)[..., None]))
        held = torch.nan_to_num(vs[tables[s][:-(-length // vc.shape[2])].long()].to(F64)).T.repeat_interleave(vc.shape[2], 1)[:, :length]
        top = (p * held[:, None, None, :]).amax(3).permute(2, 0, 1)[..., None]           # T
        off = off + seen.sum(1)[:, None, None, None] * 127 * 2.0 ** -32 * top
        out[r0:r1], slack[r0:r1] = at.flatten(1, 2), off.flatten(1, 2)
    return out, slack


def least_scale(top):
    """The least power of two, at least 2^-40, that holds `top` in 127 steps."""
    s = LEAST
    while 127 * s < top:
        s *= 2
    return s


def write(k, v, arrays, tables, lengths, starts):
    """What write() is, in 64 bits, on copies of the arrays."""
    kc, ks, vc, vs = (t.cpu().to(F64) for t in arrays)
    page = kc.shape[2]
    for x, codes, scales in ((k, kc, ks), (v, vc, vs)):
        x = x.cpu().to(F64)
        for s, length in enumerate(lengths):
            old = length - (starts[s + 1] - starts[s])
            for j in range(old // page, -(-length // page) if length > old else 0):
                p, lo, hi = int(tables[s, j]), max(old - j * page, 0), min(length - j * page, page)
                new = x[starts[s] + j * page + lo - old:starts[s] + j * page + hi - old]
                for h in range(codes.shape[1]):
                    scale = least_scale(float(new[:, h].abs().max())) if torch.isfinite(new[:, h]).all() else math.nan
                    if lo:
                        before = float(scales[p, h])
                        scale = math.nan if math.isnan(before) or math.isnan(scale) else max(before, scale)
                        if scale > before:
                            codes[p, h, :lo] = torch.round(codes[p, h, :lo] * (before / scale))
                    scales[p, h] = scale
                    codes[p, h, lo:hi] = torch.round(new[:, h] / scale) if not math.isnan(scale) else 0
    return kc.to(torch.int8), ks.float(), vc.to(torch.int8), vs.float()
