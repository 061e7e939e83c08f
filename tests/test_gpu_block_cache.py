"""Writing into the block-scaled cache, code by code and scale by scale, against its definition in 64 bits."""
import math

import pytest
import torch

from batch_helpers import BF16, fill_cache, ints, sums, tables_for, write
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import BlockCache

pytestmark = pytest.mark.gpu
F32 = torch.float32


def values(rows, heads, dim, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, heads, dim, device="cuda", generator=g) * torch.exp(2 * torch.randn(rows, heads, 1, device="cuda", generator=g))
    if rows:
        x[0::5] = 0
        x[1::7] *= 2.0 ** -60                            # under the least scale
        x[2::9, :, :1] = 127 * 2.0 ** -3                 # just held, and just not
        x[3::9, :, -1:] = -127.0625
    return x.to(dtype)


def check(cache, arrays, k, v, tables, lengths, starts):
    want = write(k, v, arrays, tables, lengths, starts)
    cache.write(k, v, tables, ints(lengths), ints(starts))
    assert cache.read_status() == 0
    for name, got, w in zip(("k codes", "k scales", "v codes", "v scales"), arrays, want):
        assert torch.equal(got.cpu().nan_to_num(-1) if got.is_floating_point() else got.cpu(), w.nan_to_num(-1) if w.is_floating_point() else w), name


@pytest.mark.parametrize("heads,dim,page,cached,new", [
    (8, 128, 16, [100], [1]), (8, 128, 16, [0], [1]), (1, 16, 16, [15], [2]), (2, 64, 32, [31, 32, 33, 0], [1, 1, 1, 40]), (3, 80, 48, [7, 0, 100], [200, 0, 49]),
    (4, 256, 64, [63, 1], [130, 64]), (8, 128, 64, [6001, 17], [300, 0]), (1, 240, 256, [255, 256, 511], [1, 300, 2]), (2, 128, 128, [0] * 40, [1] * 40), (5, 112, 16, [3] * 33, [0, 1, 30] * 11)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_against_the_definition(heads, dim, page, cached, new, dtype):
    lengths, starts = [b + m for b, m in zip(cached, new)], sums(new)
    tables, n_pages = tables_for(lengths, page)
    arrays = fill_cache(n_pages, heads, page, dim)
    rows = starts[-1]
    packed = values(rows + 3, 3 * heads, dim, dtype).unflatten(1, (3, heads))
    check(BlockCache.wrap(*arrays), arrays, packed[:, 1], packed[:, 2], tables, lengths, starts)        # three rows of padding


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_any_alignment(dtype):
    lengths, starts = [40, 21], [0, 33, 40]
    tables, n_pages = tables_for(lengths, 16)
    arrays = fill_cache(n_pages, 2, 16, 48)
    flat = values(1, 1, 50 * 2 * 51 + 1, dtype).flatten()
    k, v = (flat[o:].as_strided((40, 2, 48), (102, 51, 1)) for o in (1, 0))
    check(BlockCache.wrap(*arrays), arrays, k, v, tables, lengths, starts)


def test_token_by_token_scales_only_grow_until_the_block_begins_anew():
    heads, dim, page = 2, 64, 16
    tables, n_pages = tables_for([40], page)
    arrays = fill_cache(n_pages, heads, page, dim)
    cache = BlockCache.wrap(*arrays)
    x = values(40, heads, dim, BF16, 5)
    for i in range(40):
        check(cache, arrays, x[i:i + 1], -x[i:i + 1], tables, [i + 1], [0, 1])
    check(cache, arrays, x[:1] * 0, x[:1] * 0, tables, [17], [0, 1])                       # the second block again, from its first token
    assert float(arrays[1][int(tables[0, 1])].max()) == 2.0 ** -40


def test_scales_of_others_are_kept_where_they_suffice():
    arrays = fill_cache(3, 1, 16, 32)
    arrays[1][:], arrays[3][:] = 0.3, 0.01                # no powers of two
    tables = ints([[2]])
    x = torch.full((1, 1, 32), 3.0, device="cuda")
    check(BlockCache.wrap(*arrays), arrays, x, x, tables, [9], [0, 1])
    assert float(arrays[1][2, 0]) == pytest.approx(0.3) and float(arrays[3][2, 0]) == 2.0 ** -5


@pytest.mark.parametrize("old", [2.0 ** -50, 0.0, -1.0])
def test_scales_under_the_least_count_as_the_least(old):
    arrays = fill_cache(2, 1, 16, 32)
    codes = arrays[0][1, 0, :8].clone()
    arrays[1][:] = old
    cache = BlockCache.wrap(*arrays)
    for top, keeps in ((2.0 ** -34, 1), (2.0 ** -33, 2)):                                  # 64 and 128 steps of 2^-40
        x = torch.full((1, 1, 32), top, device="cuda")
        cache.write(x, x, ints([[1]]), ints([9]), ints([0, 1]))
        assert float(arrays[1][1, 0]) == keeps * 2.0 ** -40 and (arrays[0][1, 0, 8] == 64).all()
        assert torch.equal(arrays[0][1, 0, :8], (codes.double() / keeps).round().to(torch.int8))
    assert cache.read_status() == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_makes_its_block_and_head_nan(bad):
    arrays = fill_cache(4, 2, 16, 32)
    cache = BlockCache.wrap(*arrays)
    tables, x = ints([[1, 3]]), values(20, 2, 32, F32)
    x[3, 1, 5] = bad
    check(cache, arrays, x, x, tables, [20], [0, 20])
    assert arrays[1][1].isnan().tolist() == [False, True] and not arrays[1][3].isnan().any()
    check(cache, arrays, x[4:5], x[4:5], tables, [16], [0, 1])                             # more behind it
    assert arrays[1][1].isnan().tolist() == [False, True]
    check(cache, arrays, x[4:5], x[4:5], tables, [1], [0, 1])                              # anew
    assert not arrays[1].isnan().any()


def test_largest_and_smallest_values():
    for top in (torch.finfo(F32).max, 2.0 ** 127, 2.0 ** -33, 127 * 2.0 ** -40, 2.0 ** -45, 1e-45):
        arrays = fill_cache(1, 1, 16, 16)
        x = torch.full((2, 1, 16), top, device="cuda") * torch.linspace(-1, 1, 16, device="cuda")
        check(BlockCache.wrap(*arrays), arrays, x, -x, ints([[0]]), [2], [0, 2])


def test_what_does_not_fit_is_left_out():
    lengths, starts = [20, 40, 5], [0, 4, 8, 12]
    x = values(12, 2, 32, BF16)

    def status(tables, lengths, starts, rows=x):
        arrays = fill_cache(6, 2, 16, 32)
        was = [t.clone() for t in arrays]
        cache = BlockCache.wrap(*arrays)
        cache.write(rows, rows, ints(tables), ints(lengths), ints(starts))
        changed = sorted({int(p) for a, b in zip(arrays, was) for p in (a != b).flatten(1).any(1).nonzero()})
        return cache.read_status(), changed

    good = [[0, 1, -1], [2, 3, 4], [5, -1, -1]]
    assert status(good, lengths, starts) == (0, [1, 4, 5])
    assert status([[0, 6, -1], [2, 3, -1], [5, -1, -1]], lengths, starts) == (B.ANS_STATUS_BAD_PAGE, [5])
    assert status([[0, 1], [2, 3], [5, -1]], lengths, starts) == (B.ANS_STATUS_BAD_PAGE, [1, 5])     # 40 tokens in two pages
    assert status(good, [20, 3, 5], starts) == (B.ANS_STATUS_BAD_PAGE, [1, 5])                       # fewer tokens than new ones
    assert status(good, lengths, [0, 4, 8, 13]) == (B.ANS_STATUS_BAD_PAGE, [1, 4])
    assert status(good, lengths, [0, -4, 8, 12])[0] == B.ANS_STATUS_BAD_PAGE
    assert status(good, lengths, [0, 0, 0, 0]) == (0, [])


def test_offsets_past_32_bits():
    n_pages = (1 << 32) // (8 * 64 * 128) + 40           # codes of one array pass 4 GiB
    cache = BlockCache(n_pages, 64, 8, 128)
    x = torch.randn(3, 8, 128, device="cuda").to(BF16)
    last = n_pages - 1
    cache.write(x, -x, ints([[last]]), ints([3]), ints([0, 3]))
    got = cache.k_codes[last, :, :3].float() * cache.k_scales[last][:, None, None]
    assert (got - x.transpose(0, 1).float()).abs().max() <= cache.k_scales[last].max() / 2 and cache.read_status() == 0
    q = torch.randn(3, 8, 128, device="cuda").to(BF16)
    out = cache.attend(q, ints([[last]]), ints([3]), ints([0, 3]))
    want = -cache.k_codes[last, :, 0].float() * cache.k_scales[last][:, None]
    assert (out[0].float() - want).abs().max() <= 2.0 ** -9 * want.abs().max() + 1e-6 and cache.read_status() == 0
