"""Attention to a quantised cache on the GPU against the formula in 64 bits (attend_reference), within bounds that count roundings."""
import math

import numpy as np
import pytest
import torch

import attend_reference as ref
import quant_reference as quant

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding

    binding.lib()
    return binding


def values(cache):
    """What a cache's slots hold, [planes, slots, heads, dim] in 64 bits, from its bytes."""
    codes = quant.cache_unpack(cache.codes.cpu().numpy(), cache.dim, cache.bits)
    scales = cache.scales.view(torch.int16).cpu().numpy().view(np.uint16)
    return torch.from_numpy(quant.values(codes, scales, cache.group)).to(DEV)


class Case:
    """A cache in shuffled pages, and rows that attend to it: ``firsts`` positions held ahead of ``counts`` new ones, sequence by sequence."""

    def __init__(self, lc, kind, bits, group, heads, shared, dim, page, firsts, counts, seed=0, spread=1.0, rows_behind=2, rows_ahead=0):
        g = torch.Generator(device=DEV).manual_seed(seed + 7)
        self.kind, self.firsts, self.counts, self.page = TYPES[kind], firsts, counts, page
        used = [-(-(f + c) // page) for f, c in zip(firsts, counts)]
        width, pages = max(used + [1]) + 1, sum(used) + 2
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(used), width), -1, dtype=torch.int32, device=DEV)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = order[at : at + u]
            at += u
        slots = pages * page
        self.cache = lc.alloc_cache(slots, heads, dim, bits, group, DEV)
        kv = torch.randn(2, slots, heads, dim, generator=g, device=DEV) * torch.exp(spread * torch.randn(2, slots, heads, 1, generator=g, device=DEV))
        kv[0] += torch.randn(heads, dim, generator=g, device=DEV)
        lc.cache_write(self.cache, kv[0], kv[1], torch.arange(slots, device=DEV))
        rows = rows_ahead + sum(counts) + rows_behind
        self.q = torch.randn(rows, heads * shared, dim, generator=g, device=DEV).to(self.kind)
        begin = rows_ahead + np.concatenate([[0], np.cumsum(counts)])
        self.begin = torch.tensor(begin, dtype=torch.int32, device=DEV)
        self.first = torch.tensor(firsts, dtype=torch.int32, device=DEV)
        self.scale = 1.0 / math.sqrt(dim)

    def call(self, lc, out=None, q=None, **kw):
        if out is None:
            out = torch.full(self.q.shape, 7.0, dtype=self.kind, device=DEV)
        self.status = lc.alloc_status(DEV)
        got = lc.cache_attend(self.cache, self.q if q is None else q, self.table, self.page, self.begin, out, first=self.first, status=self.status, **kw)
        assert got is out
        return out

    def check(self, lc, got, cap=0.0, slopes=None, window=0, prefix=None, scale=None, status=0, held=None):
        held = values(self.cache) if held is None else held
        page, done = self.page, torch.zeros(got.shape[0], dtype=torch.bool, device=DEV)
        for s, (first, n) in enumerate(zip(self.firsts, self.counts)):
            at = torch.arange(first + n, device=DEV)
            place = self.table[s].long()[at // page] * page + at % page
            lo = int(self.begin[s])
            mine = slice(lo, lo + n)
            done[mine] = True
            if n == 0:
                continue
            parts = ref.attend(self.q[mine].double(), held[0][place], held[1][place], first + torch.arange(n, device=DEV), self.scale if scale is None else scale,
                               cap, slopes, window, 0 if prefix is None else int(prefix[s]))
            off, allowed = (got[mine].double() - parts[0]).abs(), ref.bound(self.kind, *parts, self.cache.dim, cap)
            assert bool((off <= allowed).all()), (s, float((off / allowed).max()), float(off.max()))
        assert bool((got[~done] == 7.0).all())  # rows of no sequence
        assert lc.last_status(self.status) == status


FEW = dict(firsts=[0, 63, 200, 5, 15], counts=[1, 1, 1, 0, 1])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("bits,group", [(4, 32), (4, 64), (4, 128), (8, 32), (8, 64), (8, 128)])
@pytest.mark.parametrize("heads,shared,dim", [(1, 1, 1), (3, 1, 49), (2, 4, 64), (1, 7, 80), (2, 3, 96), (1, 1, 100), (4, 2, 128), (2, 8, 128), (1, 2, 200), (2, 5, 256)])
def test_single_tokens(lc, kind, bits, group, heads, shared, dim):
    case = Case(lc, kind, bits, group, heads, shared, dim, 16, seed=dim, **FEW)
    case.check(lc, case.call(lc, longest=1))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("bits,group,dim", [(8, 128, 128), (4, 32, 96), (8, 64, 256)])
@pytest.mark.parametrize("counts", [[2, 3], [5, 0, 9, 1], [33, 17], [130, 64, 7], [300]])
@pytest.mark.parametrize("page", [1, 7, 64])
def test_chunks(lc, kind, bits, group, dim, counts, page):
    firsts = [0, 41, 128, 3][: len(counts)] if len(counts) > 1 else [77]
    case = Case(lc, kind, bits, group, 2, 3, dim, page, firsts, counts, seed=sum(counts), rows_ahead=3)
    case.check(lc, case.call(lc))


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("bits,group", [(4, 32), (4, 128), (8, 32), (8, 64)])
@pytest.mark.parametrize("heads,shared,dim", [(1, 1, 1), (3, 2, 49), (2, 4, 64), (1, 7, 80), (2, 3, 100), (1, 300, 40)])
def test_chunks_of_any_dim(lc, kind, bits, group, heads, shared, dim):
    """Rows that do not end on whole pieces, heads that outnumber a block's queries."""
    counts = [3] if shared > 100 else [190, 21, 64]
    case = Case(lc, kind, bits, group, heads, shared, dim, 16, [140, 0, 400][: len(counts)], counts, seed=dim)
    case.check(lc, case.call(lc))


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_long_chunks(lc, kind):
    """Chunks behind long sequences: blocks that several CTAs share, and whole ones."""
    case = Case(lc, kind, 8, 128, 2, 4, 128, 64, [9000, 300, 5000], [70, 700, 1], seed=2)
    a = case.call(lc)
    case.check(lc, a)
    assert torch.equal(a, case.call(lc, workspace=torch.full_like(lc.alloc_attend_workspace(case.cache, 3), 255)))
    case.check(lc, case.call(lc, window=1000, cap=20.0), window=1000, cap=20.0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("counts", [[1, 1, 1], [4, 6, 1], [150, 70, 9]])
@pytest.mark.parametrize("options", ["cap", "slopes", "window", "window 1", "prefix", "prefix window", "all", "scale"])
def test_options(lc, kind, counts, options):
    case = Case(lc, kind, 8, 64, 2, 4, 128, 16, [30, 500, 0], counts, seed=len(options), spread=0.5)
    kw = {}
    if options in ("cap", "all"):
        kw["cap"] = 5.0
    if options in ("slopes", "all"):
        kw["slopes"] = torch.tensor([0.5, 0.25, 0.1, 0.0, 0.01, 1.0, 2.0, 0.003], device=DEV)
    if "window" in options or options == "all":
        kw["window"] = 1 if options.endswith("1") else 70
    if "prefix" in options or options == "all":
        kw["prefix"] = torch.tensor([20, 100, 4000], dtype=torch.int32, device=DEV)
    if options == "scale":
        kw["scale"] = -0.3
    case.check(lc, case.call(lc, **kw), **kw)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("bits,group,dim,shared", [(4, 64, 128, 4), (8, 128, 128, 8), (8, 32, 80, 1), (4, 128, 256, 2)])
def test_long_and_many(lc, kind, bits, group, dim, shared):
    """Long sequences beside short ones: all SMs share them, and parts are joined."""
    r = np.random.RandomState(dim)
    firsts = [20000, 0, 3, 9000] + r.randint(0, 400, 30).tolist()
    case = Case(lc, kind, bits, group, 2, shared, dim, 64, firsts, [1] * len(firsts), seed=shared)
    a = case.call(lc, longest=1)
    case.check(lc, a)
    assert torch.equal(a, case.call(lc, longest=1))  # the same bits again
    assert torch.equal(a, case.call(lc, workspace=torch.full_like(lc.alloc_attend_workspace(case.cache, len(firsts)), 255), longest=1))  # whatever the workspace held


def test_many_sequences(lc):
    """More sequences than a CTA has threads, empty ones among them."""
    r = np.random.RandomState(3)
    n = 700
    counts, firsts = r.randint(0, 3, n).tolist(), r.randint(0, 150, n).tolist()
    case = Case(lc, "bf16", 8, 64, 1, 2, 64, 16, firsts, counts, seed=1)
    case.check(lc, case.call(lc))


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_and_no_first(lc, kind):
    case = Case(lc, kind, 8, 64, 2, 2, 64, 16, [0, 0], [9, 40], seed=4)
    joint = torch.zeros(case.q.shape[0], 4 + 3, 64 + 1, dtype=case.kind, device=DEV)
    joint[:, 2:6, 1:] = case.q
    q = joint[:, 2:6, 1:]
    out = torch.full((4, case.q.shape[0], 64 + 5), 7.0, dtype=case.kind, device=DEV)[:, :, :64].transpose(0, 1)
    status = lc.alloc_status(DEV)
    lc.cache_attend(case.cache, q, case.table, 16, case.begin, out, status=status)
    assert torch.equal(out, case.call(lc))
    case.check(lc, out)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("counts", [[1], [3], [100]])
@pytest.mark.parametrize("group", [32, 128])
def test_nan_and_inf_that_a_row_does_not_see(lc, kind, counts, group):
    """Groups with Inf and NaN behind a row, ahead of its window, or in the slots that the sequence does not use, change no bit."""
    case = Case(lc, kind, 8, group, 1, 4, 128, 16, [150], counts, seed=5)
    clean = case.call(lc, window=90)
    place = lambda p: int(case.table[0, p // 16]) * 16 + p % 16
    length = 150 + counts[0]
    hidden = [place(p) for p in range(0, 150 - 90 + 1)]
    used = {place(p) for p in range(length)}
    hidden += [s for s in range(case.cache.slots) if s not in used]
    case.cache.scales[:, hidden] = float("nan")
    assert torch.equal(clean, case.call(lc, window=90))
    case.cache.scales[:, hidden] = float("inf")
    assert torch.equal(clean, case.call(lc, window=90))
    # one behind some of the rows: those ahead of it keep their bits, those that see it are NaN where it is
    if counts[0] > 1:
        at, last = 150 + counts[0] // 2, (128 + group - 1) // group - 1
        case.cache.scales[1, place(at), :, last] = float("nan")
        got = case.call(lc, window=90)
        row = counts[0] // 2
        assert torch.equal(got[:row], clean[:row])
        assert bool(got[row : counts[0], :, group * last :].isnan().all())
        assert torch.equal(got[row : counts[0], :, : group * last], clean[row : counts[0], :, : group * last])
        case.cache.scales[0, place(at), :, last] = float("nan")
        got = case.call(lc, window=90)
        assert torch.equal(got[:row], clean[:row]) and bool(got[row : counts[0]].isnan().all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("counts", [[1], [70]])
def test_scales_of_every_size(lc, kind, counts):
    """Keys and values far smaller and larger than the type's usual numbers."""
    case = Case(lc, kind, 8, 32, 1, 2, 64, 16, [90], counts, seed=6)
    base = case.cache.scales.clone()
    for power in (-40, -20, 20 if kind != "fp16" else 6):
        case.cache.scales[1] = (base[1].float() * 2.0 ** power).to(torch.bfloat16)
        case.check(lc, case.call(lc))
    case.cache.scales[1] = base[1]
    case.cache.scales[0] = (base[0].float() * 2.0 ** -30).to(torch.bfloat16)
    case.check(lc, case.call(lc, scale=2.0 ** 30 * case.scale), scale=2.0 ** 30 * case.scale)
    # values of which a few are 2^14 times as large as the others, and hardly weigh anything
    case.cache.scales.copy_(base)
    case.cache.scales[1, ::5] = (base[1, ::5].float() * 2.0 ** -14).to(torch.bfloat16)
    case.check(lc, case.call(lc, scale=4 * case.scale), scale=4 * case.scale)


def test_bad_places(lc):
    """Pages that the cache does not have, positions beyond the table, rows that are not there: reported, nothing else is touched."""
    case = Case(lc, "bf16", 8, 64, 2, 2, 64, 16, [40, 20, 3], [1, 1, 2], seed=8)
    held = values(case.cache)
    good = case.call(lc)
    # a page number beyond the cache, one below 0, and one whose page hangs over the cache's end: its keys count as zeros
    for bad in (10 ** 9, -3, case.cache.slots // 16):
        table = case.table.clone()
        case.table[0, 1] = bad
        got = case.call(lc)
        assert lc.last_status(case.status) == lc.ERR_INDEX
        assert torch.equal(got[1:], good[1:])
        at = torch.arange(41, device=DEV)
        place = (table[0].long()[at // 16] * 16 + at % 16)
        k, v = held[0][place].clone(), held[1][place].clone()
        k[16:32] = v[16:32] = 0.0
        parts = ref.attend(case.q[:1].double(), k, v, torch.tensor([40], device=DEV), case.scale)
        assert bool(((got[:1].double() - parts[0]).abs() <= ref.bound(case.kind, *parts, 64)).all())
        case.table.copy_(table)
    for change in ("first below 0", "beyond the table", "longest", "begin", "begin ahead"):
        kw, first, begin = {}, case.first.clone(), case.begin.clone()
        rows = [1]
        if change == "first below 0":
            case.first[1] = -1
        elif change == "beyond the table":
            case.first[1] = case.table.shape[1] * 16
        elif change == "longest":
            kw["longest"], rows = 1, [2, 3]
        elif change == "begin":
            case.begin[3], rows = case.q.shape[0] + 1, [2, 3]
        else:
            case.begin[0], rows = -1, [0]
        got = case.call(lc, **kw)
        assert lc.last_status(case.status) == lc.ERR_INDEX
        for r in range(case.q.shape[0]):
            want = torch.full_like(good[r], 7.0) if r in rows else good[r]
            if not (change == "begin" and r >= 4):
                assert torch.equal(got[r], want), (change, r)
        case.first.copy_(first), case.begin.copy_(begin)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("counts", [[1], [200]])
def test_scales_and_caps_at_their_ends(lc, kind, counts):
    """A scale of 0, as small and as large as may be; a cap that leaves nothing of the scores."""
    case = Case(lc, kind, 8, 64, 1, 2, 64, 16, [90], counts, seed=7)
    for kw in (dict(scale=0.0), dict(scale=-1e-30), dict(cap=1e-38), dict(cap=1e-3), dict(scale=0.0, window=17)):
        case.check(lc, case.call(lc, **kw), **dict(kw, cap=kw.get("cap", 0.0)))
    # one key has it all: the largest score's
    got = case.call(lc, scale=1e30)
    assert bool(got[: counts[0]].isfinite().all())


def at_once(lc, cases, streams, graphs):
    outs = [torch.full(c.q.shape, 7.0, dtype=c.kind, device=DEV) for c in cases]
    works = [lc.alloc_attend_workspace(c.cache, len(c.counts)) for c in cases]
    run = lambda i: lc.cache_attend(cases[i].cache, cases[i].q, cases[i].table, cases[i].page, cases[i].begin, outs[i], first=cases[i].first, workspace=works[i])
    torch.cuda.synchronize()
    made = []
    for i, stream in enumerate(streams):
        with torch.cuda.stream(stream):
            run(i)
            if graphs:
                stream.synchronize()
                made.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(made[-1], stream=stream):
                    run(i)
    torch.cuda.synchronize()
    for turn in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                outs[i].fill_(7.0)
                made[i].replay() if graphs else run(i)
    torch.cuda.synchronize()
    return outs


@pytest.mark.parametrize("graphs", [False, True])
def test_two_at_once(lc, graphs):
    """Two calls on two streams, eagerly and as graphs, each with its workspace, give what they give alone: long chunks beside each other, and beside
    single tokens."""
    cases = [Case(lc, "bf16", 8, 64, 4, 4, 64, 16, [3000, 20], [500, 300], seed=1), Case(lc, "fp16", 4, 32, 4, 2, 64, 16, [100, 2000], [800, 1], seed=2),
             Case(lc, "bf16", 4, 64, 8, 4, 128, 64, [5000] * 9, [1] * 9, seed=3)]
    alone = [c.call(lc) for c in cases]
    outs = at_once(lc, cases, [torch.cuda.Stream() for _ in cases], graphs)
    for a, b in zip(alone, outs):
        assert torch.equal(a, b)


def test_a_captured_step_goes_by_its_buffers(lc):
    """One graph for a batch of fixed size: lengths, pages and queries change between replays."""
    case = Case(lc, "bf16", 8, 64, 2, 4, 64, 16, [200, 60, 300], [40, 1, 3], seed=9, rows_behind=0)
    out, status, work = torch.full(case.q.shape, 7.0, dtype=case.kind, device=DEV), lc.alloc_status(DEV), lc.alloc_attend_workspace(case.cache, 3)
    call = lambda: lc.cache_attend(case.cache, case.q, case.table, 16, case.begin, out, first=case.first, workspace=work, status=status)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for firsts, counts in (([200, 60, 300], [40, 1, 3]), ([0, 61, 303], [0, 1, 1]), ([190, 0, 280], [1, 20, 23]), ([100, 50, 250], [1, 1, 1])):
        case.firsts, case.counts = firsts, counts
        case.first.copy_(torch.tensor(firsts)), case.begin.copy_(torch.tensor([0] + np.cumsum(counts).tolist()))
        case.q.copy_(torch.randn(case.q.shape, device=DEV)), out.fill_(7.0)
        graph.replay()
        case.status = status
        case.check(lc, out)


def test_nothing_to_do(lc):
    cache = lc.alloc_cache(32, 2, 64, 8, 64, DEV)
    none = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    assert lc.cache_attend(cache, none, torch.zeros(1, 2, dtype=torch.int32, device=DEV), 16, torch.zeros(2, dtype=torch.int32, device=DEV)).shape == none.shape
    q = torch.ones(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    out = lc.cache_attend(cache, q, torch.zeros(0, 2, dtype=torch.int32, device=DEV), 16, torch.zeros(1, dtype=torch.int32, device=DEV))
    assert bool((out == 0).all())
    # a cache of zeros that nothing was written to: weights are equal, values 0
    out = lc.cache_attend(cache, q, torch.zeros(1, 2, dtype=torch.int32, device=DEV), 16, torch.tensor([0, 3], dtype=torch.int32, device=DEV))
    assert bool((out == 0).all())


def test_refuses(lc):
    case = Case(lc, "bf16", 8, 64, 2, 2, 64, 16, [4], [3])
    call = lambda **kw: lc.cache_attend(**dict(dict(cache=case.cache, q=case.q, table=case.table, page=16, begin=case.begin, first=case.first), **kw))
    one = lc.alloc_cache(64, 2, 64, 8, 64, DEV, planes=1)
    wide = lc.alloc_cache(64, 2, 264, 8, 64, DEV)
    for bad in (dict(q=case.q[:, :3]), dict(q=case.q[..., :63]), dict(q=case.q.double()), dict(cache=one), dict(q=case.q.cpu()), dict(table=case.table.long()),
                dict(begin=case.begin[:1]), dict(first=case.first.long()), dict(prefix=case.begin), dict(slopes=torch.ones(3, device=DEV)),
                dict(slopes=torch.ones(4, device=DEV).double()), dict(out=case.q.float()), dict(status=torch.zeros(1, device=DEV)),
                dict(q=case.q.clone().requires_grad_()), dict(workspace=torch.zeros(1 << 27, dtype=torch.uint8)), dict(workspace=torch.zeros(1 << 24, device=DEV))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(page=0), dict(window=-1), dict(longest=-1), dict(cap=-1.0), dict(cap=math.inf), dict(cap=2e30), dict(scale=math.nan), dict(scale=-2e30), dict(cache=wide, q=torch.zeros(3, 4, 264, dtype=torch.bfloat16, device=DEV)),
                dict(workspace=torch.zeros(1024, dtype=torch.uint8, device=DEV)), dict(out=case.q[:1].clone().expand(5, 4, 64))):
        with pytest.raises(lc.LCError):
            call(**bad)
    with torch.no_grad():
        call(q=case.q.clone().requires_grad_())
