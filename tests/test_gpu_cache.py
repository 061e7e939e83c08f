"""The quantised paged cache against its definition, restated with numpy's IEEE single precision (bit for bit), and
against the error that the definition allows, in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2406_06237_b200 as ans
from paper_2406_06237_b200.runtime import PagedCache

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TINY = np.float32(2.0 ** -126)


def quantise(x, bits, group):
    """x [..., dim] float32 -> codes [..., dim], scale, zero [..., dim / group]."""
    f = np.float32
    L = f((1 << bits) - 1)
    g = x.reshape(*x.shape[:-1], -1, group).astype(f)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, f(0))
    lo, hi = np.minimum(g.min(-1), f(0)), np.maximum(g.max(-1), f(0))
    u = f(1) / L
    scale = np.maximum(hi * u - lo * u, TINY)
    zero = np.minimum(np.rint(-lo / scale), L)
    code = np.clip(np.rint(g / scale[..., None]) + zero[..., None], f(0), L)
    scale = np.where(fine, scale, f("nan"))
    return code.reshape(x.shape).astype(np.uint8), scale, zero.astype(np.uint8)


def values(code, scale, zero, group, out_dtype=F32):
    """scale * (code - zero); what passes the output type's largest finite value is that value."""
    c = code.reshape(*code.shape[:-1], -1, group).astype(np.float32)
    with np.errstate(over="ignore"):
        v = ((c - zero[..., None].astype(np.float32)) * scale[..., None]).reshape(code.shape)
    most = np.float32(torch.finfo(out_dtype).max)
    return np.clip(v, -most, most)


def unpack(codes, bits):
    c = codes.cpu().numpy()
    return c if bits == 8 else np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)


def bits_of(t):
    return t.view(torch.int32 if t.dtype is F32 else torch.int16)


def same(a, b):
    """Bit for bit; NaN anywhere a NaN is."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(bits_of(a.nan_to_num(0)), bits_of(b.nan_to_num(0)))


def fill(n, heads, dim, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, heads, dim, device="cuda", generator=g) * torch.exp(2 * torch.randn(n, heads, 1, device="cuda", generator=g))
    x[0::7] = x[0::7].abs()                          # all on one side of zero
    x[3::11] = 0
    return x.to(dtype)


SHAPES = [(1, 1, 16, 16, 1, 1), (5, 8, 128, 128, 16, 3), (37, 3, 80, 80, 48, 7), (64, 2, 80, 16, 5, 20), (130, 4, 256, 256, 64, 6),
          (33, 1, 192, 96, 16, 9), (100, 5, 64, 32, 32, 8), (9, 2, 240, 240, 1, 40)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("tokens,heads,dim,group,page,pages", SHAPES)
def test_written_and_read_back(tokens, heads, dim, group, page, pages, bits, dtype):
    n_slots = pages * page
    tokens = min(tokens, n_slots)
    c = PagedCache(pages, page, heads, dim, bits, group)
    k, v = fill(tokens, heads, dim, dtype, 1), fill(tokens, heads, dim, dtype, 2)
    slots = torch.randperm(n_slots, generator=torch.Generator().manual_seed(3))[:tokens].cuda()
    c.write(k, v, slots)
    for t, codes, scales, zeros in ((k, c.k_codes, c.k_scales, c.k_zeros), (v, c.v_codes, c.v_scales, c.v_zeros)):
        code, scale, zero = quantise(t.float().cpu().numpy(), bits, group)
        at = slots.cpu().numpy()
        assert (unpack(codes, bits).reshape(n_slots, heads, dim)[at] == code).all()
        assert (scales.cpu().numpy().reshape(n_slots, heads, -1)[at] == scale).all()
        assert (zeros.cpu().numpy().reshape(n_slots, heads, -1)[at] == zero).all()
        rest = np.setdiff1d(np.arange(n_slots), at)
        assert not codes.cpu().numpy().reshape(n_slots, -1)[rest].any()      # nothing else was touched
        # the definition itself: within half a step, and half a step more where the zero-point was rounded the other way
        back = values(code, scale, zero, group).astype(np.float64)
        step = np.repeat(scale.astype(np.float64), group, -1)
        assert (np.abs(back - t.double().cpu().numpy()) <= step * (1 + 1e-5)).all()
    # read all slots as one sequence, pages in another order
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(5))
    for out_dtype in (BF16, F32):
        ko, vo = c.read(order.to(torch.int32).cuda()[None], torch.tensor([0, n_slots], dtype=torch.int32, device="cuda"), n_slots, out_dtype=out_dtype)
        where = (order[:, None] * page + torch.arange(page)).reshape(-1).numpy()
        for out, codes, scales, zeros in ((ko, c.k_codes, c.k_scales, c.k_zeros), (vo, c.v_codes, c.v_scales, c.v_zeros)):
            want = values(unpack(codes, bits).reshape(n_slots, heads, dim)[where], scales.cpu().numpy().reshape(n_slots, heads, -1)[where],
                          zeros.cpu().numpy().reshape(n_slots, heads, -1)[where], group)
            assert same(out.cpu(), torch.from_numpy(want).to(out_dtype))
    assert c.read_status() == 0


@pytest.mark.parametrize("bits", [8, 4])
def test_sequences(bits):
    """Ragged sequences, empty ones among them, through tables with unused entries that name no page."""
    page, heads, dim = 16, 2, 64
    lengths = [0, 1, 16, 17, 0, 100, 33, 0]
    need = [-(-n // page) for n in lengths]
    c = PagedCache(sum(need) + 2, page, heads, dim, bits)
    order = torch.randperm(sum(need) + 2, generator=torch.Generator().manual_seed(1)).tolist()
    tables = torch.full((len(lengths), 9), -1, dtype=torch.int32)
    slots, at = [], 0
    for i, n in enumerate(lengths):
        for j in range(need[i]):
            tables[i, j] = order[at]; at += 1
        slots += [int(tables[i, p // page]) * page + p % page for p in range(n)]
    total = sum(lengths)
    k, v = fill(total, heads, dim, BF16, 7), fill(total, heads, dim, BF16, 8)
    c.write(k, v, torch.tensor(slots, device="cuda"))
    starts = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()
    wide = torch.full((len(lengths), 20), -5, dtype=torch.int32, device="cuda")
    wide[:, 4:13] = tables.cuda()
    for t in (tables.cuda(), wide[:, 4:13]):
        ko, vo = c.read(t, starts, total)
        for out, x in ((ko, k), (vo, v)):
            want = values(*quantise(x.float().cpu().numpy(), bits, dim), dim)
            assert same(out.cpu(), torch.from_numpy(want).to(BF16))
    # buffers longer than the sequences: the rest stays
    ko = torch.full((total + 40, heads, dim), 9.0, device="cuda")
    vo = ko.clone()
    c.read(tables.cuda(), starts, k_out=ko, v_out=vo)
    assert (ko[total:] == 9).all() and (vo[total:] == 9).all() and not (ko[:total] == 9).all()
    assert c.read_status() == 0


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_inputs(bits, dtype):
    """Slices of one product's output, at aligned and odd places, heads in another order of strides."""
    tokens, heads, dim = 21, 4, 64
    qkv = torch.randn(tokens, 3 * heads * dim + 5, device="cuda").to(dtype)
    pairs = [(qkv[:, heads * dim:2 * heads * dim].unflatten(1, (heads, dim)), qkv[:, 2 * heads * dim:3 * heads * dim].unflatten(1, (heads, dim))),
             (qkv[:, 1:1 + heads * dim].unflatten(1, (heads, dim)), qkv[:, 3:3 + heads * dim].unflatten(1, (heads, dim))),
             (torch.randn(heads, tokens, dim, device="cuda").to(dtype).transpose(0, 1), torch.randn(1, 1, dim, device="cuda").to(dtype).expand(tokens, heads, dim))]
    for k, v in pairs:
        c, d = PagedCache(2, 16, heads, dim, bits), PagedCache(2, 16, heads, dim, bits)
        slots = torch.arange(tokens, device="cuda") + 3
        c.write(k, v, slots)
        d.write(k.contiguous(), v.contiguous(), slots)
        for f in ("k_codes", "k_scales", "k_zeros", "v_codes", "v_scales", "v_zeros"):
            assert torch.equal(getattr(c, f), getattr(d, f)), f


@pytest.mark.parametrize("bits", [8, 4])
def test_values_at_the_limits(bits):
    """Zeros, constants, the type's largest and smallest values, NaN and infinities: groups by themselves."""
    big = float(torch.finfo(BF16).max)
    rows = [[0.0], [5.0], [-5.0], [big, -big], [big], [1e-40, -1e-40], [float("nan"), 1.0], [float("inf"), 1.0], [-float("inf")], [1e-30, 1.0], [-3.0, -0.0]]
    x = torch.tensor([(r * 16)[:16] for r in rows])[:, None, :].cuda()
    for dtype in (BF16, F32):
        t = x.to(dtype)
        c = PagedCache(1, len(rows), 1, 16, bits)
        c.write(t, t, torch.arange(len(rows), device="cuda"))
        ko, vo = c.read(torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([0, len(rows)], dtype=torch.int32, device="cuda"), len(rows), out_dtype=F32)
        want = values(*quantise(t.float().cpu().numpy(), bits, 16), 16)
        assert same(ko.cpu(), torch.from_numpy(want)) and same(vo.cpu(), torch.from_numpy(want))
        half, _ = c.read(torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([0, len(rows)], dtype=torch.int32, device="cuda"), len(rows))
        assert same(half.cpu(), torch.from_numpy(values(*quantise(t.float().cpu().numpy(), bits, 16), 16, BF16)).to(BF16))
        bad = ~t.isfinite().all(-1)[:, 0]
        assert ko[bad].isnan().all() and ko[~bad].isfinite().all()
        assert (ko[0] == 0).all() and ((ko[1] - 5).abs() <= 1e-5).all() and ((ko[2] + 5).abs() <= 1e-5).all()


def test_slots_and_pages_outside():
    c = PagedCache(4, 8, 2, 32, 8)
    k = fill(5, 2, 32, BF16, 1)
    before = c.k_codes.clone()
    c.write(k, k, torch.tensor([-1, 32, 1 << 40, -(1 << 40), 31], device="cuda"))
    assert c.read_status() == ans.ANS_STATUS_BAD_PAGE and c.read_status() == 0
    assert torch.equal(c.k_codes.view(32, -1)[:31], before.view(32, -1)[:31]) and c.k_codes.view(32, -1)[31].any()
    c.write(k, k, torch.full((5,), -1, device="cuda"))
    assert c.read_status() == 0                      # skipped tokens are no fault
    starts = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    for table, zero in (([[3, 4, 3]], slice(8, 16)), ([[3, -1, 3]], slice(8, 16)), ([[3, 3]], slice(16, 20))):
        ko, vo = c.read(torch.tensor(table, dtype=torch.int32, device="cuda"), starts, 20)
        assert c.read_status() == ans.ANS_STATUS_BAD_PAGE
        assert (ko[zero] == 0).all() and (vo[zero] == 0).all() and ko[7].any()
    ko, _ = c.read(torch.tensor([[3, 3, 3]], dtype=torch.int32, device="cuda"), starts, 10)
    assert c.read_status() == ans.ANS_STATUS_BAD_PAGE and ko[7].any() and not ko[8].any()


def test_a_cache_past_four_gigabytes():
    """Codes whose byte offsets pass 32 bits."""
    page, heads, dim = 64, 8, 256
    pages = (1 << 32) // (page * heads * dim) + 2
    c = PagedCache(pages, page, heads, dim, 8)
    k, v = fill(3, heads, dim, BF16, 1), fill(3, heads, dim, BF16, 2)
    slots = torch.tensor([0, (pages - 1) * page + 5, (pages - 2) * page + 63], device="cuda")
    c.write(k, v, slots)
    tables = torch.tensor([[0, pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    ko, vo = c.read(tables, torch.tensor([0, 192], dtype=torch.int32, device="cuda"), 192)
    for out, x in ((ko, k), (vo, v)):
        want = torch.from_numpy(values(*quantise(x.float().cpu().numpy(), 8, dim), dim)).to(BF16)
        assert same(out[[0, 64 + 5, 128 + 63]].cpu(), want)
    assert c.read_status() == 0


def test_empty():
    c = PagedCache(2, 4, 1, 16)
    e = torch.empty(0, 1, 16, device="cuda").to(BF16)
    c.write(e, e, torch.empty(0, dtype=torch.int64, device="cuda"))
    ko, vo = c.read(torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 0)
    assert ko.shape == (0, 1, 16)
    ko, vo = c.read(torch.empty(2, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), 0)
    assert c.read_status() == 0


def test_on_a_stream_and_in_a_graph():
    c = PagedCache(4, 16, 2, 64, 4)
    k, v = fill(40, 2, 64, BF16, 1), fill(40, 2, 64, BF16, 2)
    slots = torch.arange(40, device="cuda")
    tables, starts = torch.arange(3, dtype=torch.int32, device="cuda")[None].contiguous(), torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.write(k, v, slots)
        c.read(tables, starts, k_out=ko, v_out=vo)
    k.copy_(fill(40, 2, 64, BF16, 5))
    g.replay()
    torch.cuda.synchronize()
    for out, x in ((ko, k), (vo, v)):
        assert same(out.cpu(), torch.from_numpy(values(*quantise(x.float().cpu().numpy(), 4, 64), 64)).to(BF16))


def test_refusals():
    c = PagedCache(2, 4, 2, 32)
    k = torch.randn(3, 2, 32, device="cuda").to(BF16)
    slots = torch.arange(3, device="cuda")
    for bad in ((k[:, :1], k, slots), (k, k.float(), slots), (k, k, slots.int()), (k, k, slots[:2]), (k.half(), k.half(), slots), (k.cpu(), k, slots),
                (k.transpose(1, 2), k, slots)):
        with pytest.raises(ValueError):
            c.write(*bad)
    t, s = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    for kw in (dict(), dict(rows=3, k_out=k), dict(k_out=k, v_out=k.float()), dict(k_out=k[:, :1], v_out=k[:, :1]), dict(rows=5, k_out=k, v_out=k)):
        with pytest.raises(ValueError):
            c.read(t, s, **kw)
    for bad in ((t.long(), s), (t, s.long()), (t, s[:1]), (t[0], s)):
        with pytest.raises(ValueError):
            c.read(*bad, 3)
    for kw in (dict(bitwidth=3), dict(group=24), dict(head_dim=0), dict(n_pages=0)):
        with pytest.raises(ValueError):
            PagedCache(**{**dict(n_pages=2, page_size=4, heads=2, head_dim=32), **kw})
    odd = PagedCache(2, 4, 1, 8)                     # groups of 8: not a size that the kernels take
    with pytest.raises(ans.AnsError):
        odd.write(k[:, :1, :8], k[:, :1, :8], slots)
    with pytest.raises(RuntimeError):
        PagedCache(2, 4, 2, 32, device="cpu")
    with pytest.raises(ValueError):
        PagedCache.wrap(c.k_codes, c.k_scales, c.k_zeros, c.v_codes, c.v_scales[:1], c.v_zeros, 8)
