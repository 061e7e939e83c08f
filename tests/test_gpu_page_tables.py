"""Block tables and slot maps against a loop over the requests' tokens."""
import random

import pytest
import torch

from batch_helpers import INT, ints, sums
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import Batch, PagedCache, PageTables

pytestmark = pytest.mark.gpu


def plan(cached, new, page, tables, free, taken, rows):
    tables = [list(r) for r in tables]
    slots, positions = [], []
    for i, (b, m) in enumerate(zip(cached, new)):
        for j in range(-(-b // page), -(-(b + m) // page)):
            tables[i][j] = free[taken]
            taken += 1
        slots += [tables[i][p // page] * page + p % page for p in range(b, b + m)]
        positions += range(b, b + m)
    rest = rows - len(slots)
    lengths = [b + m for b, m in zip(cached, new)]
    return tables, Batch(sums(new), lengths, sums(lengths), slots + [-1] * rest, positions + [0] * rest, [taken])


def case(seed, n, page, most_new, most_cached, wide=2):
    rng = random.Random(seed)
    cached = [rng.choice((0, 1, page - 1, page, rng.randint(0, most_cached))) for _ in range(n)]
    new = [rng.choice((0, 1, 1, rng.randint(0, most_new))) for _ in range(n)]
    pages = max((-(-(b + m) // page) for b, m in zip(cached, new)), default=0) + wide
    held = [-(-b // page) for b in cached]
    n_pages = sum(held) + sum(-(-(b + m) // page) - h for b, m, h in zip(cached, new, held)) + 9
    order = list(range(n_pages))
    rng.shuffle(order)
    taken, tables = 4, []
    pool = order[:]
    for h in held:
        tables.append([pool.pop() for _ in range(h)] + [-5] * (pages - h))
    free = [-9] * taken + pool
    return cached, new, tables, free, taken


def same(got, want):
    for name, g, w in zip(Batch._fields, got, want):
        assert g.tolist() == w, name


@pytest.mark.parametrize("n,page,most_new,most_cached,room", [
    (1, 16, 1, 100, 0), (1, 1, 5, 3, 3), (3, 16, 40, 100, 0), (64, 16, 1, 1500, 5), (512, 48, 9, 300, 0), (513, 64, 30, 100, 77), (1500, 16, 20, 60, 1),
    (4096, 32, 6, 90, 0), (7, 16, 9000, 10, 0), (2, 128, 40000, 70000, 1000), (1, 16, 0, 50, 4), (40, 7, 700, 33, 0)])
def test_against_a_loop(n, page, most_new, most_cached, room):
    cached, new, tables, free, taken = case(n + page, n, page, most_new, most_cached)
    rows = sum(new) + room
    f = PageTables(page)
    t = ints(tables)
    got = f(t, ints(cached), ints(new), ints(free), ints([taken]), rows=rows)
    want_tables, want = plan(cached, new, page, tables, free, taken, rows)
    same(got, want)
    assert t.tolist() == want_tables and f.read_status() == 0
    again = f(ints(tables), ints(cached), ints(new), ints(free), ints([taken]), out=got)
    assert again is got
    same(got, want)


def test_a_loop_in_place_in_a_graph():
    n, page, rows = 5, 16, 8
    f = PageTables(page)
    cached, new, taken = ints([0, 15, 16, 30, 7]), ints([1, 1, 1, 0, 3]), ints([2])
    tables, free = ints([[-1] * 6, [40, -1, -1, -1, -1, -1], [41] + [-1] * 5, [42, 43, -1, -1, -1, -1], [44] + [-1] * 5]), ints([-1, -1, *range(30)])
    out = f.buffers(n, rows)._replace(lengths=cached, taken=taken)
    start = (cached.tolist(), tables.tolist())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f(tables, cached, new, free, taken, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(tables, cached, new, free, taken, out=out)
    now, lists, at = start[0], start[1], 2
    for step in range(6):
        if step == 3:
            new.copy_(ints([2, 0, 0, 1, 1]))
        m = [1, 1, 1, 0, 3] if step < 3 else [2, 0, 0, 1, 1]
        if step:
            graph.replay()
        lists, want = plan(now, m, page, lists, [-1, -1, *range(30)], at, rows)
        now, at = want.lengths, want.taken[0]
        same(out, want)
        assert tables.tolist() == lists
    assert f.read_status() == 0


@pytest.mark.parametrize("change", ["free", "table", "rows", "new", "cached", "taken", "sum"])
def test_what_does_not_fit_is_left_alone(change):
    cached, new, free, taken, rows, pages = [20, 0, 31], [5, 40, 1], list(range(10, 20)), 0, 46, 4
    if change == "free": free = free[:2]
    if change == "table": pages = 2
    if change == "rows": rows = 45
    if change == "new": new[1] = -1
    if change == "cached": cached[0] = -3
    if change == "taken": taken = 11
    if change == "sum": cached = [2 ** 31 - 3, 2 ** 31 - 2, 31]
    tables = [[1, 2, -1, -1], [-1] * 4, [3, 4, -1, -1]]
    f = PageTables(16)
    t = ints(tables)[:, :pages]
    got = f(t, ints(cached), ints(new), ints(free), ints([taken]), rows=rows)
    assert f.read_status() == B.ANS_STATUS_BAD_PAGE
    assert t.tolist() == [r[:pages] for r in tables] and got.lengths.tolist() == cached and got.taken.tolist() == [taken]
    assert got.starts.tolist() == [0] * 4 and got.slots.tolist() == [-1] * rows and got.positions.tolist() == [0] * rows


def test_a_page_that_is_none_gives_no_slot():
    f = PageTables(16)
    got = f(ints([[-1, 3]]), ints([10]), ints([8]), ints([7]), ints([0]), rows=8)
    assert f.read_status() == B.ANS_STATUS_BAD_PAGE
    assert got.slots.tolist() == [-1] * 6 + [7 * 16, 7 * 16 + 1]


def test_slots_and_ends_serve_the_paged_cache():
    cached, new, tables, free, taken = case(3, 6, 16, 30, 50)
    f, rows = PageTables(16), sum(new)
    t = ints(tables)
    cache = PagedCache(max(max(free), max(map(max, tables))) + 1, 16, 2, 64)
    first = f(t, torch.zeros(6, dtype=INT, device="cuda"), ints([0] * 6), ints(free), ints([taken]), rows=0)
    assert first.ends.tolist() == [0] * 7
    got = f(t, ints(cached), ints(new), ints(free), ints([taken]), rows=rows)
    k = torch.randn(rows, 2, 64, device="cuda")
    cache.write(k, -k, got.slots)
    back, _ = cache.read(t, got.ends, rows=int(got.ends[-1]), out_dtype=torch.float32)
    for s in range(6):
        e, m = int(got.ends[s + 1]), new[s]
        assert (back[e - m:e] - k[got.starts[s]:got.starts[s + 1]]).abs().max() < 0.05 if m else True
    assert cache.read_status() == 0


def test_a_batch_without_requests_still_has_its_sums():
    f = PageTables(16)
    none, (starts, ends, taken) = ints([]), (ints([5]) for _ in range(3))
    out = Batch(starts, none, ends, torch.empty(0, dtype=torch.int64, device="cuda"), none, taken)
    f(torch.zeros(0, 4, dtype=INT, device="cuda"), none, none, ints([3, 1, 2]), ints([2]), out=out)
    assert f.read_status() == 0
    same(out, Batch([0], [], [0], [], [], [2]))
