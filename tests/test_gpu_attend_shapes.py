"""Attention in forms that take other kernels: divided tiles of every width of head, codes past 32 bits under tiles, a captured call whose
prompts change, and rows of few queries at the accuracy that their kernel has."""
import pytest
import torch

from batch_helpers import BF16, F64, attention, fill_cache, ints, sums, tables_for, values_of
from operator_helpers import rounds_from
from paper_2406_06237_b200.runtime import BlockCache

pytestmark = pytest.mark.gpu


def queries(rows, heads, dim, seed=2):
    return torch.randn(rows, heads, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(BF16)


@pytest.mark.parametrize("heads,share,dim,page,cached,new", [
    (2, 8, 64, 64, [3000], [64]), (1, 4, 256, 32, [4000], [70]), (2, 8, 80, 16, [2500, 40], [50, 60]), (1, 4, 240, 32, [3000], [40]), (1, 5, 48, 16, [5000], [77]),
    (2, 2, 256, 64, [1500, 9], [100, 100]), (1, 64, 128, 64, [2000], [1])])
@pytest.mark.parametrize("how", [dict(), dict(window=700), dict(causal=False)])
def test_divided_tiles(heads, share, dim, page, cached, new, how):
    lengths, starts = [b + m for b, m in zip(cached, new)], sums(new)
    tables, n_pages = tables_for(lengths, page)
    arrays, q = fill_cache(n_pages, heads, page, dim), queries(starts[-1] + 3, heads * share, dim)
    cache, out = BlockCache.wrap(*arrays), torch.full_like(q, 7.0)
    cache.attend(q, tables, ints(lengths), ints(starts), out=out, **how)
    want, slack = attention(q, arrays, tables, lengths, starts, **how)
    n = starts[-1]
    assert rounds_from(out[:n], want[:n], slack[:n]).all() and (out[n:] == 7).all() and cache.read_status() == 0


def test_tiles_of_codes_past_32_bits():
    n_pages = (1 << 32) // (8 * 64 * 128) + 40           # codes of one array pass 4 GiB
    cache = BlockCache(n_pages, 64, 8, 128)
    new, last = 150, n_pages - 1
    tables = ints([[last, 3, last - 2]])
    x = queries(new, 16, 128, 5)
    cache.write(x[:, :8], x[:, 8:], tables, ints([new]), ints([0, new]))
    q = queries(new, 8, 128)
    out = cache.attend(q, tables, ints([new]), ints([0, new]))
    held = ints([[2, 0, 1]])
    arrays = [t[[3, last - 2, last]] for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    want, slack = attention(q, arrays, held, [new], [0, new])
    assert rounds_from(out, want, slack).all() and cache.read_status() == 0


def test_a_graph_serves_prompts_of_other_lengths():
    heads, dim, page, rows = 2, 128, 32, 500
    arrays = fill_cache(120, heads, page, dim)
    cache, q = BlockCache.wrap(*arrays), queries(rows, heads * 4, dim)
    tables = torch.randperm(120, device="cuda", generator=torch.Generator("cuda").manual_seed(0)).to(torch.int32)[:90].view(3, 30)
    lengths, starts, out = ints([400, 200, 300]), ints([0, 400, 401, 480]), torch.zeros_like(q)
    cache.attend(q, tables, lengths, starts, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, tables, lengths, starts, out=out)
    for length, start in (([400, 200, 300], [0, 400, 401, 480]), ([1, 950, 0], [0, 1, 480, 480]), ([60, 900, 13], [0, 30, 33, 46]), ([900, 5, 5], [0, 500, 500, 500])):
        lengths.copy_(ints(length))
        starts.copy_(ints(start))
        out.fill_(7.0)
        graph.replay()
        want, slack = attention(q, arrays, tables, length, start)
        n = start[-1]
        assert rounds_from(out[:n], want[:n], slack[:n]).all() and (out[n:] == 7).all()
    assert cache.read_status() == 0


@pytest.mark.parametrize("share,dim,cached,new", [(1, 64, 500, 1), (4, 128, 3000, 1), (8, 128, 700, 2), (2, 256, 900, 3)])
def test_few_queries_keep_small_weights(share, dim, cached, new):
    """Where the tokens with large weights have values of 0, what is left is made of small weights.  Few queries round P_i = 2^14 p_i c_i / T (c_i the
    scale of the token's values, T the largest p_j c_j) to fp16, so that one under 2^-14 is off by 2^-25 at most and its term by
    2^-25 * 127 * T / 2^14 = 127 * 2^-39 T, where the common bound of attention() has 127 * 2^-32 T for both kernels."""
    page, length = 16, cached + new
    tables, n_pages = tables_for([length], page)
    arrays, q = fill_cache(n_pages, 1, page, dim), queries(new, share, dim)
    arrays[0][:] = (arrays[0].float() * 0.5).round().to(torch.int8)
    top = tables[0, 2].long()
    arrays[0][top, 0] = q[0, 0].float().sign().to(torch.int8) * 100                     # tokens that a row looks at most
    arrays[2][top], arrays[1][:], arrays[3][:] = 0, 2.0 ** -5, 2.0 ** -3
    cache = BlockCache.wrap(*arrays)
    got = cache.attend(q, tables, ints([length]), ints([0, new]), longest=new, scale=0.11)
    want, slack = attention(q, arrays, tables, [length], [0, new], scale=0.11)
    k = values_of(*arrays[:2], tables[0], length)[0]
    score = torch.einsum("tjd,sd->tjs", q.to(F64), k) * 0.11
    later = torch.arange(length, device="cuda") > torch.arange(cached, length, device="cuda")[:, None]
    p = score.masked_fill(later[:, None], -torch.inf).softmax(2)
    coarse = (~later).sum(1)[:, None, None] * 127 * (p * 2.0 ** -3).amax(2)[..., None]  # of which slack holds 2^-32
    assert rounds_from(got, want, slack - coarse * (2.0 ** -32 - 2.0 ** -39)).all() and cache.read_status() == 0
