"""Attention where the scales of the values lie anywhere in the range that the cache's write can choose, 2^-40 to 2^122."""
import pytest
import torch

from batch_helpers import BF16, attention, fill_cache, ints, sums, tables_for
from operator_helpers import rounds_from
from paper_2406_06237_b200.runtime import BlockCache

pytestmark = pytest.mark.gpu

# heads, share, dim, page, cached, new: few queries whole and divided, tiles whole and divided, every width of head
CASES = [(2, 4, 128, 16, [100], [1]), (2, 4, 128, 16, [3000, 40], [1, 1]), (2, 2, 128, 16, [700], [90]), (1, 4, 128, 64, [3000], [40]), (2, 1, 64, 16, [900], [3]),
         (1, 8, 64, 32, [2500], [40]), (1, 3, 256, 16, [500], [2]), (1, 2, 256, 16, [2100], [70])]


def check(arrays, q, tables, lengths, starts, **kw):
    cache = BlockCache.wrap(*arrays)
    got = cache.attend(q, tables, ints(lengths), ints(starts), **kw)
    assert cache.read_status() == 0
    want, slack = attention(q, arrays, tables, lengths, starts, **kw)
    ok = rounds_from(got, want, slack)
    assert ok.all(), (int((~ok).sum()), ok.numel())


def case(heads, share, dim, page, cached, new):
    lengths, starts = [b + m for b, m in zip(cached, new)], sums(new)
    tables, n_pages = tables_for(lengths, page)
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(starts[-1], heads * share, dim, device="cuda", generator=g).to(BF16)
    return fill_cache(n_pages, heads, page, dim), q, tables, lengths, starts, g


@pytest.mark.parametrize("shape", CASES)
@pytest.mark.parametrize("low,high", [(110, 122), (-40, 110), (-40, 121)])
@pytest.mark.parametrize("how", [dict(), dict(window=50)])
def test_any_scale_that_the_write_makes(shape, low, high, how):
    arrays, q, tables, lengths, starts, g = case(*shape)
    arrays[3].copy_(torch.exp2(torch.randint(low, high, arrays[3].shape, device="cuda", generator=g).float()))
    check(arrays, q, tables, lengths, starts, **how)
    arrays[3].mul_(1.37)                                 # and between them
    check(arrays, q, tables, lengths, starts, **how)


@pytest.mark.parametrize("shape", CASES)
@pytest.mark.parametrize("first", [True, False])
def test_pages_of_zeros_beside_very_large_values(shape, first):
    """A page of zeros has the least scale.  Its tokens count in the sum of the weights as all others do, whether they come before
    the large ones or behind them."""
    arrays, q, tables, lengths, starts, _ = case(*shape)
    page = shape[3]
    arrays[3][:] = 2.0 ** 115
    for s, n in enumerate(lengths):
        held = tables[s, :-(-n // page)].long()
        zeros = held[:len(held) // 2] if first else held[len(held) // 2:]
        arrays[2][zeros], arrays[3][zeros] = 0, 2.0 ** -40
    check(arrays, q, tables, lengths, starts)


@pytest.mark.parametrize("new", [1, 90])
def test_what_write_makes_of_the_largest_values(new):
    page, n = 16, 64 + new
    cache = BlockCache(n // page + 1, page, 1, 64)
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(n, 1, 64, device="cuda", generator=g)
    v = torch.randn(n, 1, 64, device="cuda", generator=g).clamp(-3, 3) * 2.0 ** 125
    tables = ints([list(range(n // page + 1))])
    cache.write(k, v, tables, ints([n]), ints([0, n]))
    q = torch.randn(new, 2, 64, device="cuda", generator=g).to(BF16)
    got = cache.attend(q, tables, ints([n]), ints([0, new]))
    assert cache.read_status() == 0
    want, slack = attention(q, (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), tables, [n], [0, new])
    assert rounds_from(got, want, slack).all() and (got != 0).any()
