"""Attention over the block-scaled cache against its definition in 64 bits."""
import math

import pytest
import torch

from batch_helpers import BF16, attention, fill_cache, ints, sums, tables_for
from operator_helpers import rounds_from
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import BlockCache

pytestmark = pytest.mark.gpu


def queries(rows, heads, dim, seed=2, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn(rows, heads, dim, device="cuda", generator=g)).to(BF16)


def check(arrays, q, tables, lengths, starts, **kw):
    cache = BlockCache.wrap(*arrays)
    longest = kw.pop("longest", None)
    out = torch.full_like(q, 7.0)
    got = cache.attend(q, tables, ints(lengths), ints(starts), longest=longest, out=out, **kw)
    assert got is out and cache.read_status() == 0
    want, slack = attention(q, arrays, tables, lengths, starts, **kw)
    n = starts[-1]
    ok = rounds_from(out[:n], want[:n], slack[:n])
    assert ok.all(), (int((~ok).sum()), ok.numel(), float(((out[:n].double() - want[:n]).abs() / slack[:n].clamp(min=1e-30)).max()))
    assert (out[n:] == 7.0).all()
    return out


CASES = [                                                # heads, share, dim, page, cached, new
    (8, 4, 128, 16, [100], [1]), (1, 1, 64, 16, [0], [1]), (2, 1, 128, 64, [700], [1]), (1, 8, 128, 64, [5000], [1]), (2, 7, 80, 48, [300, 15, 16, 0], [1, 1, 1, 1]),
    (1, 16, 128, 16, [130, 127, 128], [1, 1, 1]), (2, 3, 256, 32, [400, 33], [1, 2]), (1, 5, 16, 16, [20], [3]), (4, 2, 112, 128, [1000, 0, 250], [1, 5, 0]),
    (2, 4, 128, 16, [0, 200, 31], [70, 33, 17]), (1, 8, 64, 32, [90], [100]), (3, 1, 128, 64, [0], [300]), (2, 2, 256, 16, [10, 600], [150, 129]),
    (1, 128, 128, 16, [60], [1]), (1, 40, 64, 16, [260], [2]), (2, 4, 96, 256, [2000] * 3, [1, 260, 3]), (8, 4, 128, 16, [int(700 / (i + 1)) for i in range(30)], [1] * 30),
    (1, 4, 128, 64, [0], [1025]), (2, 8, 128, 64, [3000], [64]),
]


@pytest.mark.parametrize("heads,share,dim,page,cached,new", CASES)
@pytest.mark.parametrize("how", [dict(), dict(window=1), dict(window=100), dict(causal=False), dict(causal=False, window=70)])
def test_against_the_definition(heads, share, dim, page, cached, new, how):
    lengths, starts = [b + m for b, m in zip(cached, new)], sums(new)
    tables, n_pages = tables_for(lengths, page)
    arrays = fill_cache(n_pages, heads, page, dim)
    q = queries(starts[-1] + 2, heads * share, dim)
    longest = max(new) if len(new) % 2 else None
    check(arrays, q, tables, lengths, starts, longest=longest, **how)


@pytest.mark.parametrize("new", [1, 40])
def test_longest_that_is_wrong_changes_nothing(new):
    tables, n_pages = tables_for([300 + new, 20 + new], 16)
    arrays = fill_cache(n_pages, 2, 16, 64)
    q = queries(2 * new, 8, 64)
    for longest in (1, 3, 2 * new, 100000):
        check(arrays, q, tables, [300 + new, 20 + new], [0, new, 2 * new], longest=longest)


@pytest.mark.parametrize("new", [1, 50])
def test_rows_that_see_nothing_are_zero(new):
    arrays = fill_cache(9, 2, 16, 64)
    tables = ints([[0, 1, 2, 3], [4, 5, 6, 7]])
    out = check(arrays, queries(2 * new, 4, 64), tables, [0, 5], [0, new, 2 * new])          # fewer tokens than new ones
    assert (out[:new] == 0).all() and (out[new:2 * new - 5] == 0).all()
    out = check(arrays, queries(2 * new, 4, 64), tables, [0, 5], [0, new, 2 * new], causal=False)
    assert (out[:new] == 0).all() and (out[new:] != 0).any()


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("low,high", [(-20, 20), (-40, -30), (60, 100)])
def test_scales_of_very_different_blocks(new, low, high):
    lengths = [700 + new]
    tables, n_pages = tables_for(lengths, 16)
    arrays = fill_cache(n_pages, 2, 16, 128)
    g = torch.Generator(device="cuda").manual_seed(1)
    arrays[3].copy_(torch.exp2(torch.randint(low, high, arrays[3].shape, device="cuda", generator=g).float()))
    check(arrays, queries(new, 4, 128), tables, lengths, [0, new])
    arrays[3].mul_(1.37)                                 # and of no powers of two
    check(arrays, queries(new, 4, 128), tables, lengths, [0, new])


@pytest.mark.parametrize("new", [1, 90])
def test_sharp_and_flat_rows(new):
    lengths = [2000 + new]
    tables, n_pages = tables_for(lengths, 64)
    arrays = fill_cache(n_pages, 1, 64, 128)
    for size, scale in ((30.0, None), (1e-3, None), (2.0 ** 100, 2.0 ** -103), (2.0 ** -110, 2.0 ** 109), (1.0, 0.0), (1.0, -0.1), (3.0, 2.0)):
        q = queries(new, 4, 128, size=size)
        q[:, 1] = 0
        check(arrays, q, tables, lengths, [0, new], scale=scale)


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("which", [1, 3])
def test_a_nan_block_is_seen_only_by_rows_that_see_it(new, which):
    page, lengths = 16, [200 + new]
    tables, n_pages = tables_for(lengths, page)
    arrays = fill_cache(n_pages, 2, page, 64)
    cache, q = BlockCache.wrap(*arrays), queries(new, 4, 64)
    clean = cache.attend(q, tables, ints(lengths), ints([0, new]), window=20)
    last = (200 + new - 1) // page                       # the last page: hidden from none but the rows before it
    arrays[which][int(tables[0, 0]), :] = math.nan       # hidden by the window
    arrays[which][int(tables[0, last]), 1] = math.nan
    got = cache.attend(q, tables, ints(lengths), ints([0, new]), window=20)
    sees = torch.arange(200, 200 + new, device="cuda") >= last * page
    assert got[sees][:, 2:].isnan().all() and torch.equal(got[:, :2], clean[:, :2]) and torch.equal(got[~sees], clean[~sees])


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_that_is_not_finite_stays_in_its_row(new, bad):
    lengths = [100 + new, 300 + new]
    tables, n_pages = tables_for(lengths, 16)
    arrays = fill_cache(n_pages, 2, 16, 64)
    cache, q = BlockCache.wrap(*arrays), queries(2 * new, 8, 64)
    clean = cache.attend(q, tables, ints(lengths), ints([0, new, 2 * new]))
    q[new // 2, 3, 5] = bad
    got = cache.attend(q, tables, ints(lengths), ints([0, new, 2 * new]))
    assert got[new // 2, 3].isnan().all()
    got[new // 2, 3] = clean[new // 2, 3]
    assert torch.equal(got, clean) and cache.read_status() == 0


def test_strides_alignment_and_in_place():
    lengths, starts = [70, 300], [0, 5, 40]
    tables, n_pages = tables_for(lengths, 16)
    arrays = fill_cache(n_pages, 2, 16, 64)
    cache = BlockCache.wrap(*arrays)
    packed = queries(40, 24, 64).unflatten(1, (3, 8))
    want = check(arrays, packed[:, 1].contiguous(), tables, lengths, starts)
    assert torch.equal(cache.attend(packed[:, 1], tables, ints(lengths), ints(starts)), want)
    flat = torch.zeros(40 * 8 * 64 + 3, dtype=BF16, device="cuda")
    off = flat[3:].view(40, 8, 64)
    off.copy_(packed[:, 1])
    assert torch.equal(cache.attend(off, tables, ints(lengths), ints(starts)), want)
    wide = torch.zeros(40, 8, 66, dtype=BF16, device="cuda")[:, :, :64]
    assert torch.equal(cache.attend(packed[:, 1], tables, ints(lengths), ints(starts), out=wide), want)
    own = packed[:, 1].clone()
    assert cache.attend(own, tables, ints(lengths), ints(starts), out=own) is own and torch.equal(own, want)
    assert cache.read_status() == 0


def test_results_do_not_vary_and_a_graph_serves_other_lengths():
    page, n = 16, 12
    tables, n_pages = tables_for([900] * n, page)
    arrays = fill_cache(n_pages, 4, page, 128)
    cache, q = BlockCache.wrap(*arrays), queries(n, 16, 128)
    lengths, starts = ints([900 - 70 * i for i in range(n)]), ints(range(n + 1))
    want = cache.attend(q, tables, lengths, starts, longest=1)
    for _ in range(5):
        assert torch.equal(cache.attend(q, tables, lengths, starts, longest=1), want)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, tables, lengths, starts, longest=1, out=out)
    graph.replay()
    assert torch.equal(out, want)
    lengths.copy_(ints([1 + 80 * i for i in range(n)]))
    graph.replay()
    assert torch.equal(out, cache.attend(q, tables, lengths, starts, longest=1))
    want, slack = attention(q, arrays, tables, lengths.tolist(), list(range(n + 1)))
    assert rounds_from(out, want, slack).all() and cache.read_status() == 0


@pytest.mark.parametrize("dim,window", [(128, 1024), (64, 300), (256, 500), (128, 0)])
def test_long_prompts_again_and_again(dim, window):
    """Warps of a tile that are at different blocks: rows whose window hides a block rescale while others go on."""
    new, page = [1635 - 62 * i for i in range(13)], 64
    lengths, starts = [m + 2 * i for i, m in enumerate(new)], sums(new)
    tables, n_pages = tables_for(lengths, page)
    arrays = fill_cache(n_pages, 2, page, dim, spread=12)
    cache, q = BlockCache.wrap(*arrays), queries(starts[-1], 14, dim, size=3.0)
    a, b = ints(lengths), ints(starts)
    want = cache.attend(q, tables, a, b, window=window)
    for _ in range(40):
        assert torch.equal(cache.attend(q, tables, a, b, window=window), want)
    assert cache.read_status() == 0
    for s in (0, 12):                                    # the first and the last of them against the definition
        r0, r1 = starts[s], starts[s + 1]
        exact, slack = attention(q[r0:r1], arrays, tables[s:s + 1], lengths[s:s + 1], [0, r1 - r0], window=window)
        assert rounds_from(want[r0:r1], exact, slack).all()


def test_pages_outside_the_cache_count_as_not_there():
    arrays = fill_cache(6, 2, 16, 64)
    cache, q = BlockCache.wrap(*arrays), queries(41, 4, 64)
    for new in (1, 41):
        good = cache.attend(q[:new], ints([[0, 1, 2, 3]]), ints([48]), ints([0, new]), causal=False)
        assert cache.read_status() == 0
        got = cache.attend(q[:new], ints([[0, 1, 2, 6]]), ints([64]), ints([0, new]), causal=False)
        assert cache.read_status() == B.ANS_STATUS_BAD_PAGE and torch.equal(got, good)
        got = cache.attend(q[:new], ints([[0, 1, 2]]), ints([64]), ints([0, new]), causal=False)
        assert cache.read_status() == B.ANS_STATUS_BAD_PAGE and torch.equal(got, good)
        got = cache.attend(q[:new], ints([[-1, -1, -1, 9]]), ints([64]), ints([0, new]), causal=False)
        assert cache.read_status() == B.ANS_STATUS_BAD_PAGE and (got == 0).all()


def test_nothing_to_do():
    cache = BlockCache(4, 16, 2, 64)
    q = queries(3, 4, 64)
    out = torch.full_like(q, 3.0)
    cache.attend(q, ints([[0]]), ints([5]), ints([0, 0]), out=out)
    assert (out == 3).all()
    assert cache.attend(q[:0], ints([[0]]), ints([5]), ints([0, 0])).shape == (0, 4, 64)
    assert cache.attend(q, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), ints([]), ints([0]), out=out) is out and (out == 3).all()
    cache.write(q[:, :2], q[:, 2:], ints([[0]]), ints([5]), ints([0, 0]))
    assert cache.read_status() == 0


def test_another_stream():
    tables, n_pages = tables_for([400, 90], 16)
    arrays = fill_cache(n_pages, 2, 16, 128)
    q = queries(2, 8, 128)
    cache = BlockCache.wrap(*arrays)
    want = cache.attend(q, tables, ints([400, 90]), ints([0, 1, 2]))
    side = torch.cuda.Stream()
    lengths, starts = ints([400, 90]), ints([0, 1, 2])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = cache.attend(q, tables, lengths, starts)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("new", [[1, 1], [3, 90]])
def test_room_that_is_too_small_is_refused(new):
    lengths, starts = [3000, 4000], sums(new)
    tables, n_pages = tables_for(lengths, 16)
    cache = BlockCache.wrap(*fill_cache(n_pages, 2, 16, 128))
    cache.attend(queries(starts[-1], 8, 128), tables, ints(lengths), ints(starts))
    torch.cuda.synchronize()
    d, b = cache._attend, cache._attend_batch
    need = B.ans_attend_room_bytes(cache._desc, b, d)
    assert need and d.room_bytes == need
    d.room_bytes = need - 1
    with pytest.raises(B.AnsError) as e:
        B.ans_attend(cache._desc, b, d, cache._status)
    assert e.value.code == B.ANS_ERR_BUFFER_TOO_SMALL
    d.room_bytes, d.d_room = need, None
    with pytest.raises(B.AnsError) as e:
        B.ans_attend(cache._desc, b, d, cache._status)
    assert e.value.code == B.ANS_ERR_BUFFER_TOO_SMALL


def test_more_query_heads_than_the_border():
    new, lengths = [1, 0, 7, 1], [500, 30, 7, 1]
    tables, n_pages = tables_for(lengths, 32)
    check(fill_cache(n_pages, 1, 32, 64), queries(sum(new), 40, 64), tables, lengths, sums(new))
