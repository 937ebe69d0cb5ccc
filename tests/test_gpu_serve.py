"""From a checkpoint to a step of a served layer: a chain of streams recovered into 4-bit weights, products with them, what they give
written into a quantised cache, and a batch of sequences read back, all on one stream without a wait in between."""
import numpy as np
import pytest
import torch

import quant_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bits,group", [(8, 64), (4, 32)])
def test_recover_multiply_write_read(oracle, bits, group):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding as lc

    heads, dim, cols, page, steps = 3, 64, 320, 4, 9
    rows = 2 * heads * dim  # the projections of keys and values, one above the other
    g = torch.Generator(device=DEV).manual_seed(bits)
    base = torch.randn(rows * cols, generator=g, device=DEV) * 0.05
    tracked, cur, streams = base.clone(), base.clone(), []
    for _ in range(2):
        cur = cur + torch.randn(rows * cols, generator=g, device=DEV) * 1e-3
        s, tracked = lc.compress_update(tracked, cur, 4)
        streams.append(s.clone())

    q4, ws = lc.alloc_q4(rows, cols, group, DEV), lc.alloc_workspace(0, DEV)
    lc.recover_q4_async(base, streams, q4, torch.empty_like(base), ws)
    # three sequences that grow at different paces: -1 where one has ended
    lengths, width = [9, 4, 6], 3
    table = torch.randperm(9, generator=g, device=DEV).to(torch.int32).view(3, width)
    cache, status = lc.alloc_cache(9 * page, heads, dim, bits, group, DEV), lc.alloc_status(DEV)
    x = torch.randn(steps, 3, cols, generator=g, device=DEV).to(torch.bfloat16)
    given = []
    for t in range(steps):
        kv = lc.q4_matvec(q4, x[t]).view(3, 2, heads, dim)
        slots = torch.where(torch.tensor([t < n for n in lengths], device=DEV), table[:, t // page].long() * page + t % page, -1)
        lc.cache_write(cache, kv[:, 0], kv[:, 1], slots, status)
        given.append(kv)
    begin = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device=DEV)
    outs = [torch.zeros(sum(lengths), heads, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    lc.cache_read_pages(cache, table, page, begin, outs, status=status)
    assert lc.last_status(ws) == lc.OK and lc.last_status(status) == lc.OK

    # the weights: exactly the recovered state's codes
    state = oracle.recover(base.cpu().numpy(), [s.cpu().numpy() for s in streams]).reshape(rows, cols).astype(np.float64)
    codes, scales = ref.quantize(state, 4, group)
    w = ref.values(codes, scales, group)
    given = torch.stack(given)  # [step, sequence, plane, head, dim]
    xd = x.double().cpu().numpy()
    want, size = xd @ w.T, np.abs(xd) @ np.abs(w).T
    got = given.double().cpu().numpy().reshape(steps, 3, rows)
    bound = size * (17 * group / 16 * 2.0 ** -23 + (cols / group + 16) * 2.0 ** -24) + np.abs(want) * 2.0 ** -8 * 1.001
    assert np.all(np.abs(got - want) <= bound)
    # the cache: what each step gave, quantised once
    for plane in range(2):
        seq = torch.cat([given[:n, s, plane] for s, n in enumerate(lengths)])
        codes, scales = ref.quantize(seq.double().cpu().numpy(), bits, group)
        assert torch.equal(outs[plane].cpu(), torch.from_numpy(ref.values(codes, scales, group)).float().to(torch.bfloat16))


def test_two_streams_and_two_graphs_at_once():
    """Products, writes and reads of two states on two streams, eagerly and as graphs replayed side by side, give what they give alone."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding as lc

    g = torch.Generator(device=DEV).manual_seed(3)
    sides = []
    for rows, cols, tokens, bits in ((3000, 2100, 2, 8), (500, 9000, 5, 4)):
        w = torch.randn(rows, cols, generator=g, device=DEV)
        q4, ws = lc.alloc_q4(rows, cols, 64, DEV), lc.alloc_workspace(0, DEV)
        x, y = torch.randn(tokens, cols, generator=g, device=DEV), torch.empty(tokens, rows, device=DEV)
        cache, status = lc.alloc_cache(96, 2, 80, bits, 32, DEV), lc.alloc_status(DEV)
        kv = torch.randn(48, 2, 2, 80, generator=g, device=DEV)
        at, outs = torch.randperm(96, generator=g, device=DEV)[:48], [torch.empty(48, 2, 80, device=DEV) for _ in range(2)]

        def run(w=w, q4=q4, ws=ws, x=x, y=y, cache=cache, status=status, kv=kv, at=at, outs=outs):
            lc.q4_quantize_async(w, q4, ws)
            lc.q4_matvec(q4, x, y)
            lc.cache_write(cache, kv[:, 0], kv[:, 1], at, status)
            lc.cache_read(cache, at, outs, status=status)

        run()
        torch.cuda.synchronize()
        sides.append((run, [y, *outs], [t.clone() for t in (y, *outs)], (ws, status)))

    streams = [torch.cuda.Stream(DEV) for _ in sides]

    def compare():
        torch.cuda.synchronize()
        for _, got, want, words in sides:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            assert all(lc.last_status(word) == lc.OK for word in words)
            for t in got:
                t.zero_()
        torch.cuda.synchronize()

    compare()
    for _ in range(20):
        for (run, *_), s in zip(sides, streams):
            with torch.cuda.stream(s):
                run()
    compare()
    graphs = [torch.cuda.CUDAGraph() for _ in sides]
    for (run, *_), s, graph in zip(sides, streams, graphs):
        with torch.cuda.graph(graph, stream=s):
            run()
    for _ in range(20):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    compare()
