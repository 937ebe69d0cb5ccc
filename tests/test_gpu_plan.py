"""The plan of a step on the GPU against the text: pages, slots and books, whole or not at all."""
import numpy as np
import pytest
import torch

import attend_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding

    binding.lib()
    return binding


def books(n, page, longest, most, seed, extra=3, ends=0.15):
    r = np.random.RandomState(seed)
    held = r.randint(0, longest + 1, n)
    tokens = r.randint(0, most + 1, n)
    tokens[r.rand(n) < ends] = -r.randint(1, 5)
    width = -(-(longest + most) // page)
    has, wants = -(-held // page), -(-(held + np.maximum(tokens, 0)) // page)
    pages = int(has.sum() + (wants - has).sum()) + extra
    order = r.permutation(pages).astype(np.int32)
    table, at = np.full((n, width), -7, np.int32), 0
    for s in range(n):
        table[s, : has[s]] = order[at : at + has[s]]
        at += has[s]
    spare = np.full(pages, -9, np.int32)
    spare[: pages - at] = order[at:]
    return held, tokens, table, spare, pages - at


def on_device(lc, held, table, spare, count, page, stride=0):
    t = lambda x: torch.tensor(np.asarray(x, np.int32), device=DEV)
    wide = torch.full((table.shape[0], table.shape[1] + stride), 77, dtype=torch.int32, device=DEV)
    wide[:, : table.shape[1]] = t(table)
    return lc.Pages(wide[:, : table.shape[1]], t(held), t(spare), t([count]), page), wide


def same(got, want):
    return got.cpu().numpy().tolist() == list(np.asarray(want).tolist())


@pytest.mark.parametrize("n,page,longest,most,room", [(1, 16, 0, 1, 0), (1, 1, 5, 40, 3), (48, 16, 900, 1, 5), (300, 7, 60, 9, 0), (513, 64, 300, 70, 1000), (1025, 16, 50, 2, 9),
                                                      (2048, 100, 20, 90, 1), (5000, 3, 9, 4, 0)])
@pytest.mark.parametrize("in_place", [True, False])
def test_steps(lc, n, page, longest, most, room, in_place):
    held, tokens, table, spare, count = books(n, page, longest, most, n + page)
    rows = int(np.maximum(tokens, 0).sum()) + room
    want = ref.plan(table, held, spare, count, tokens, page, rows)
    assert want is not None
    pages, wide = on_device(lc, held, table, spare, count, page, stride=3)
    given = torch.tensor(tokens.astype(np.int32), device=DEV)
    plan, status = lc.alloc_plan(pages, rows, in_place), lc.alloc_status(DEV)
    for again in range(1 if in_place else 2):  # books that go elsewhere: the same step once more
        for t in (plan.begin, plan.first, plan.slots):
            t.fill_(-55)
        assert lc.cache_plan(pages, given, plan=plan, status=status) is plan
        for got, x in zip((plan.begin, plan.first, plan.slots, plan.held, plan.count), want[:5]):
            assert same(got, x if isinstance(x, list) else [x])
        assert same(pages.table, want[5]) and same(pages.spare, want[6])
        assert bool((wide[:, -3:] == 77).all())
    if not in_place:
        assert same(pages.held, held) and same(pages.count, [count])
    assert lc.last_status(status) == lc.OK


def test_many_steps_keep_the_books(lc):
    """Sequences come, grow and end for 60 steps: the books are those of the text, and no page is ever in two places."""
    r = np.random.RandomState(5)
    n, page, width, total = 40, 4, 12, 300
    pages = lc.alloc_pages(n, width, total, page, DEV)
    status = lc.alloc_status(DEV)
    held, table, spare, count = np.zeros(n, int), np.zeros((n, width), np.int32), np.arange(total - 1, -1, -1).astype(np.int32), total
    for step in range(60):
        tokens = r.randint(0, 4, n)
        tokens[r.rand(n) < 0.1] = -1
        tokens[held + tokens > width * page] = -1
        rows = 200
        want = ref.plan(table, held, spare, count, tokens, page, rows)
        plan = lc.cache_plan(pages, torch.tensor(tokens.astype(np.int32), device=DEV), rows=rows, status=status)
        begin, first, slots, held, count, table, spare = want
        held = np.array(held)
        assert same(plan.slots, slots) and same(plan.begin, begin) and same(plan.first, first) and same(pages.held, held) and same(pages.count, [count])
        used = [table[s, j] for s in range(n) for j in range(-(-held[s] // page))] + spare[:count].tolist()
        assert sorted(used) == list(range(total))
        assert same(pages.table, table)
    assert lc.last_status(status) == lc.OK


@pytest.mark.parametrize("n", [3, 700])
@pytest.mark.parametrize("fault", ["pages", "rows", "width", "held", "held below 0", "count", "count below 0", "list"])
def test_what_does_not_fit_changes_nothing(lc, n, fault):
    page = 8
    held, tokens, table, spare, count = books(n, page, 100, 9, 11, extra=0, ends=0.0)
    tokens[0], rows, code = 5, int(tokens.sum()) + 5, lc.ERR_CAPACITY
    spare = np.concatenate([spare, np.arange(4, dtype=np.int32)])
    if fault == "pages":
        wanted = int((-(-(held + tokens) // page) - -(-held // page)).sum())
        assert wanted > 0
        count = wanted - 1
    elif fault == "rows":
        rows = int(tokens.sum()) - 1
    elif fault == "width":
        tokens[n // 2] = table.shape[1] * page - held[n // 2] + 1
        rows += 10000
    elif fault == "list":
        tokens[1], held[1], count, code = -1, 30, len(spare) - 1, lc.ERR_INDEX
    else:
        code = lc.ERR_INDEX
        if fault == "held":
            held[n - 1] = table.shape[1] * page + 1
        elif fault == "held below 0":
            held[n - 1] = -1
        else:
            count = len(spare) + 1 if fault == "count" else -1
    pages, _ = on_device(lc, held, table, spare, count, page)
    for in_place in (False, True):
        plan, status = lc.alloc_plan(pages, rows, in_place), lc.alloc_status(DEV)
        lc.cache_plan(pages, torch.tensor(tokens.astype(np.int32), device=DEV), plan=plan, status=status)
        assert lc.last_status(status) == code
        assert same(plan.begin, [0] * (n + 1)) and bool((plan.slots == -1).all())
        assert same(plan.held, held) and same(plan.count, [count]) and same(pages.table, table) and same(pages.spare, spare)


def test_a_page_that_is_not_there(lc):
    pages, _ = on_device(lc, [3, 5], np.array([[9, -1], [1, 0]], np.int32), np.array([2, -1, -1], np.int32), 1, 4)
    status = lc.alloc_status(DEV)
    plan = lc.cache_plan(pages, torch.tensor([2, 1], dtype=torch.int32, device=DEV), rows=3, status=status)
    assert same(plan.slots, [-1, 8, 1]) and lc.last_status(status) == lc.ERR_INDEX


def test_captured(lc):
    """A step that advances the books, captured once and replayed: like as many calls."""
    n, page = 20, 16
    pages = lc.alloc_pages(n, 10, 150, page, DEV)
    tokens = torch.ones(n, dtype=torch.int32, device=DEV)
    plan, status = lc.alloc_plan(pages, n + 4), lc.alloc_status(DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.cache_plan(pages, tokens, plan=plan, status=status)
    held, table, spare, count = np.zeros(n, int), np.zeros((n, 10), np.int32), pages.spare.cpu().numpy(), 150
    r = np.random.RandomState(2)
    for step in range(12):
        now = r.randint(-1, 2, n)
        tokens.copy_(torch.tensor(now.astype(np.int32)))
        graph.replay()
        begin, first, slots, held, count, table, spare = ref.plan(table, held, spare, count, now, page, n + 4)
        assert same(plan.slots, slots) and same(plan.begin, begin) and same(plan.first, first) and same(pages.held, held) and same(pages.count, [count])
    assert lc.last_status(status) == lc.OK
