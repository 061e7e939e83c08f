"""Page tables whose lengths and place in the free list are written over what was read, by one block and by clusters of 2, 4 and 8."""
import pytest
import torch

from batch_helpers import ints
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import PageTables
from test_gpu_page_tables import case, plan, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,page,most_new,most_cached,room", [
    (1, 16, 2000, 100, 2100), (40, 16, 300, 100, 2100), (300, 16, 40, 900, 4200), (512, 48, 60, 300, 9000), (513, 64, 3, 100, 0), (513, 64, 50, 100, 9000),
    (1500, 16, 3, 60, 1), (1500, 16, 40, 60, 5000), (4096, 32, 1, 90, 0), (4096, 32, 20, 90, 77), (7, 16, 9000, 10, 9000), (2, 128, 40000, 70000, 1000)])
@pytest.mark.parametrize("over", ["both", "lengths", "taken"])
def test_over_what_was_read(n, page, most_new, most_cached, room, over):
    cached, new, tables, free, taken = case(n + page, n, page, most_new, most_cached)
    rows = sum(new) + room
    want_tables, want = plan(cached, new, page, tables, free, taken, rows)
    f = PageTables(page)
    t, c, at = ints(tables), ints(cached), ints([taken])
    was = [x.clone() for x in (t, c, at)]
    new, free = ints(new), ints(free)
    out = f.buffers(n, rows)
    out = out._replace(**{k: v for k, v in (("lengths", c), ("taken", at)) if over in ("both", k)})
    for _ in range(5):
        for x, y in zip((t, c, at), was):
            x.copy_(y)
        for x in out:
            if x is not c and x is not at:
                x.fill_(-3)
        assert f(t, c, new, free, at, out=out) is out
        same(out, want)
        assert t.tolist() == want_tables
    assert f.read_status() == 0


@pytest.mark.parametrize("n,rows", [(1, 9000), (600, 5000), (4096, 2)])
def test_what_does_not_fit_is_left_alone_in_place(n, rows):
    f = PageTables(16)
    c, new, at, free = ints([20 + i % 3 for i in range(n)]), ints([1] * n), ints([0]), ints(range(30))
    new[n // 2] = 30 * 16 * n + 5                        # more than there are pages
    was, t = c.clone(), torch.full((n, 4), 3, dtype=torch.int32, device="cuda")
    out = f.buffers(n, rows)._replace(lengths=c, taken=at)
    f(t, c, new, free, at, out=out)
    assert f.read_status() == B.ANS_STATUS_BAD_PAGE
    assert torch.equal(c, was) and at.tolist() == [0] and (t == 3).all() and (out.slots == -1).all() and (out.starts == 0).all()
    assert torch.equal(out.ends[1:], was.cumsum(0).to(torch.int32))
