"""Steps of a served layer: a plan, keys and values written to its slots, attention, with sequences that begin, grow, are checked in drafts and end, eagerly and
as a graph that is replayed; against the same in 64 bits on lists that the test keeps."""
import math

import numpy as np
import pytest
import torch

import attend_reference as ref
import quant_reference as quant

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("kind,bits,group", [(torch.bfloat16, 8, 64), (torch.float16, 4, 32)])
def test_steps(captured, kind, bits, group):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding as lc

    heads, shared, dim, page, n, rows, width = 2, 3, 64, 4, 5, 120, 60
    r = np.random.RandomState(bits)
    g = torch.Generator(device=DEV).manual_seed(bits)
    pages = lc.alloc_pages(n, width, 200, page, DEV)
    cache = lc.alloc_cache(200 * page, heads, dim, bits, group, DEV)
    plan, status, work = lc.alloc_plan(pages, rows), lc.alloc_status(DEV), lc.alloc_attend_workspace(cache, n)
    tokens = torch.zeros(n, dtype=torch.int32, device=DEV)
    q = torch.zeros(rows, heads * shared, dim, dtype=kind, device=DEV)
    kv = torch.zeros(rows, 2 * heads, dim, dtype=kind, device=DEV)
    out = torch.zeros_like(q)

    def step():
        lc.cache_plan(pages, tokens, plan=plan, status=status)
        lc.cache_write(cache, kv[:, :heads], kv[:, heads:], plan.slots, status)
        lc.cache_attend(cache, q, pages.table, page, plan.begin, out, first=plan.first, workspace=work, status=status)

    graph = None
    if captured:
        step()  # no tokens: nothing changes
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    kept = [[np.zeros((0, heads, dim)), np.zeros((0, heads, dim))] for _ in range(n)]
    for turn in range(14):
        new = np.array([r.choice([0, 1, 1, 5, 30]) for _ in range(n)])
        for s in range(n):
            if len(kept[s][0]) + new[s] > 180 or (turn == 9 and s == 2):
                new[s] = -1
        while np.maximum(new, 0).sum() > rows:
            new[new.argmax()] = 1
        tokens.copy_(torch.tensor(new.astype(np.int32)))
        q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        kv.copy_(torch.randn(kv.shape, generator=g, device=DEV))
        out.fill_(7.0)
        graph.replay() if captured else step()
        row, given = 0, kv.double().cpu().numpy()
        for s in range(n):
            m = max(0, int(new[s]))
            if new[s] < 0:
                kept[s] = [np.zeros((0, heads, dim)), np.zeros((0, heads, dim))]
            for i in range(2 if m else 0):
                x = given[row : row + m, i * heads : (i + 1) * heads]
                kept[s][i] = np.concatenate([kept[s][i], quant.values(*quant.quantize(x, bits, group), group)])
            if m:
                k, v = (torch.from_numpy(x).to(DEV) for x in kept[s])
                positions = len(kept[s][0]) - m + torch.arange(m, device=DEV)
                parts = ref.attend(q[row : row + m].double(), k, v, positions, 1.0 / math.sqrt(dim))
                assert bool(((out[row : row + m].double() - parts[0]).abs() <= ref.bound(kind, *parts, dim)).all()), (turn, s)
            row += m
        assert bool((out[row:] == 7.0).all())
        assert pages.held.tolist() == [len(x[0]) for x in kept]
    assert lc.last_status(status) == lc.OK
