"""Pages that the window has left behind may be given back: what their entries of the table hold is no one's concern."""
import pytest
import torch

from batch_helpers import BF16, attention, fill_cache, ints, sums, tables_for
from operator_helpers import rounds_from
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import BlockCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 32, 48, 64, 256])
@pytest.mark.parametrize("heads,share,dim,cached,new", [(2, 4, 128, [1000, 333], [1, 1]), (1, 2, 64, [777], [5]), (2, 2, 128, [1000], [90]), (1, 8, 128, [3001], [40]),
                                                        (1, 4, 256, [500, 90], [30, 1])])
@pytest.mark.parametrize("window", [1, 60, 100, 300])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_before_the_window(page, heads, share, dim, cached, new, window, causal):
    lengths, starts = [b + m for b, m in zip(cached, new)], sums(new)
    tables, n_pages = tables_for(lengths, page)
    arrays = fill_cache(n_pages, heads, page, dim)
    q = torch.randn(starts[-1], heads * share, dim, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(BF16)
    want, slack = attention(q, arrays, tables, lengths, starts, causal=causal, window=window)
    for s, n in enumerate(lengths):
        first = max((cached[s] + 1 if causal else n) - window, 0)                      # that a row sees
        tables[s, :first // page] = -1
    cache = BlockCache.wrap(*arrays)
    got = cache.attend(q, tables, ints(lengths), ints(starts), causal=causal, window=window)
    assert cache.read_status() == 0
    assert rounds_from(got, want, slack).all()
    tables[0, max((cached[0] + 1 if causal else lengths[0]) - window, 0) // page] = n_pages       # one that is seen
    cache.attend(q, tables, ints(lengths), ints(starts), causal=causal, window=window)
    assert cache.read_status() == B.ANS_STATUS_BAD_PAGE
