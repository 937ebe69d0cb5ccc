"""The quantised cache on the GPU against the text in 64 bits (quant_reference): what a write leaves in the cache, byte for byte, and what
reads return, through slots and through pages."""
import numpy as np
import pytest
import torch

import quant_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def lc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding

    binding.lib()
    return binding


def rows_of(n, heads, dim, kind, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, heads, dim, generator=g, device=DEV) * torch.exp(torch.randn(n, heads, 1, generator=g, device=DEV))
    return x.to(TYPES[kind])


def expected(x, bits, group):
    """(codes, scale bits, values) of rows."""
    codes, scales = ref.quantize(x.double().cpu().numpy(), bits, group)
    return codes, scales, torch.from_numpy(ref.values(codes, scales, group)).to(torch.float32)


def check_slots(cache, plane, slots, codes, scales):
    held = cache.codes[plane].cpu().numpy()[slots]
    assert np.array_equal(ref.cache_unpack(held, cache.dim, cache.bits), codes)
    assert np.array_equal(cache.scales[plane].view(torch.int16).cpu().numpy().view(np.uint16)[slots], scales)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("heads,dim", [(1, 1), (2, 7), (3, 49), (4, 80), (8, 128), (2, 300)])
def test_write_and_read(lc, bits, group, kind, heads, dim):
    n, slots = 37, 101
    cache = lc.alloc_cache(slots, heads, dim, bits, group, DEV)
    cache.codes.fill_(0xA5)
    cache.scales.fill_(3.0)
    before = cache.codes.clone(), cache.scales.clone()
    k, v = rows_of(n, heads, dim, kind, 1), rows_of(n, heads, dim, kind, 2)
    at = torch.randperm(slots, device=DEV)[:n]
    at[5] = at[20] = -1  # two rows that fill the batch up
    status = lc.alloc_status(DEV)
    lc.cache_write(cache, k, v, at, status)
    place = at.cpu().numpy()
    real = np.flatnonzero(place >= 0)
    for plane, x in ((0, k), (1, v)):
        codes, scales, _ = expected(x, bits, group)
        check_slots(cache, plane, place[real], codes[real], scales[real])
    free = np.setdiff1d(np.arange(slots), place)
    for now, then in zip((cache.codes, cache.scales), before):
        assert torch.equal(now[:, free], then[:, free])  # nothing else was touched
    # back, in every type; rows without a slot stay
    for out in TYPES.values():
        outs = [torch.full((n, heads, dim), 5.0, dtype=out, device=DEV) for _ in range(2)]
        got = lc.cache_read(cache, at, outs, status=status)
        for x, y in zip((k, v), got):
            want = expected(x, bits, group)[2].to(out)
            want[[5, 20]] = 5.0
            assert torch.equal(y.cpu(), want)
    assert lc.last_status(status) == lc.OK


@pytest.mark.parametrize("bits", [4, 8])
def test_borders_inf_nan_and_zeros(lc, bits):
    top = 2 ** (bits - 1) - 1
    r = np.random.RandomState(bits)
    x = np.zeros((12, 1, 64), np.float32)
    x[1, 0] = r.randint(-2 * top, 2 * top + 1, 64) / 2
    x[1, 0, [0, 32]] = top  # scale 1: halves are borders
    x[2, 0] = np.nextafter(x[1, 0], np.float32(0))
    x[2, 0, [0, 32]] = top
    x[3] = x[1] * np.float32(1.9921875)
    x[4] = x[1] * np.float32(2.0 ** -126)
    x[5] = r.randint(-5, 6, 64) * np.float32(2.0 ** -149)
    x[6] = r.uniform(-3.4e38, 3.4e38, 64)
    x[7] = r.randn(64)
    x[8] = r.randn(64)
    x[9] = r.randn(64)
    x[7, 0, 3], x[8, 0, 40], x[9, 0, 63] = np.inf, np.nan, -np.inf
    x[10] = top * (1 + (2 * r.randint(0, 64) + 1) * 2.0 ** -9)  # between two scales
    t = torch.from_numpy(x).to(DEV)
    cache = lc.alloc_cache(12, 1, 64, bits, 32, DEV, planes=1)
    at = torch.arange(12, device=DEV)
    lc.cache_write(cache, t, None, at)
    codes, scales, values = expected(t, bits, 32)
    check_slots(cache, 0, np.arange(12), codes, scales)
    got = lc.cache_read(cache, at, dtype=torch.float32)[0].cpu()
    assert torch.equal(got.nan_to_num(nan=1e9), values.nan_to_num(nan=1e9)) and int(got.isnan().sum()) == 3 * 32


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides(lc, kind):
    # keys and values side by side behind something else in the rows of one tensor, at an odd offset; heads ahead of rows in the output
    n, heads, dim = 19, 3, 64
    joint = rows_of(n, 3 * heads + 1, dim + 1, kind, 3)
    k, v = joint[:, heads : 2 * heads, 1:], joint[:, 2 * heads : 3 * heads, :dim]
    cache = lc.alloc_cache(64, heads, dim, 8, 64, DEV)
    at = torch.randperm(64, device=DEV)[:n]
    lc.cache_write(cache, k, v, at)
    outs = [torch.zeros(heads, n, dim + 3, dtype=TYPES[kind], device=DEV)[:, :, :dim].transpose(0, 1) for _ in range(2)]
    assert lc.cache_read(cache, at, outs) is outs
    for x, y in zip((k, v), outs):
        assert torch.equal(y.cpu(), expected(x, 8, 64)[2].to(TYPES[kind]))
    # one row for all, as a broadcast gives it
    lc.cache_write(cache, k[:1].expand(n, heads, dim), v[:1].expand(n, heads, dim), at)
    got = lc.cache_read(cache, at, dtype=TYPES[kind])[0]
    assert torch.equal(got.cpu(), expected(k[:1].expand(n, heads, dim), 8, 64)[2].to(TYPES[kind]))


@pytest.mark.parametrize("page", [1, 16, 100])
@pytest.mark.parametrize("bits,group,heads,dim", [(4, 32, 2, 80), (8, 128, 4, 128)])
def test_pages(lc, page, bits, group, heads, dim):
    lengths, first = [0, 1, 33, 0, 100, 101, 16, 0], [0, 99, 5, 3, 100, 0, 17, 0]
    width = -(-201 // page)
    pages = len(lengths) * width + 2
    cache = lc.alloc_cache(pages * page, heads, dim, bits, group, DEV)
    k, v = rows_of(pages * page, heads, dim, "bf16", 4), rows_of(pages * page, heads, dim, "bf16", 5)
    lc.cache_write(cache, k, v, torch.arange(pages * page, device=DEV))
    wide = torch.randperm(pages, device=DEV).to(torch.int32)[: len(lengths) * width].view(len(lengths), width)
    table = torch.full((len(lengths), width + 3), -7, dtype=torch.int32, device=DEV)[:, :width]
    table.copy_(wide)
    status = lc.alloc_status(DEV)
    for starts in (None, first):
        begin = np.concatenate([[2], 2 + np.cumsum(lengths)])
        total = int(begin[-1])
        place = []
        for s, n in enumerate(lengths):
            p = np.arange(n) + (starts[s] if starts else 0)
            place.append(wide.cpu().numpy()[s][p // page].astype(np.int64) * page + p % page)
        place = np.concatenate(place)
        outs = [torch.full((total + 4, heads, dim), 9.0, dtype=torch.float16, device=DEV) for _ in range(2)]
        lc.cache_read_pages(cache, table, page, torch.tensor(begin, dtype=torch.int32, device=DEV), outs,
                            None if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV), status)
        for x, y in zip((k, v), outs):
            want = torch.full((total + 4, heads, dim), 9.0, dtype=torch.float16)
            want[2:total] = expected(x[torch.from_numpy(place).to(DEV)], bits, group)[2].half()
            assert torch.equal(y.cpu(), want)  # rows ahead of the first sequence and behind the last are as they were
    assert lc.last_status(status) == lc.OK


def test_slots_and_pages_that_do_not_exist(lc):
    heads, dim, page = 2, 40, 8
    cache = lc.alloc_cache(64, heads, dim, 8, 32, DEV)
    k, v = rows_of(64, heads, dim, "fp32", 6), rows_of(64, heads, dim, "fp32", 7)
    lc.cache_write(cache, k, v, torch.arange(64, device=DEV))
    before = cache.codes.clone(), cache.scales.clone()
    for bad in (64, -2, 1 << 40, -(1 << 62)):
        at = torch.tensor([bad, -1], device=DEV)
        for fn in (lambda s: lc.cache_write(cache, k[:2], v[:2], at, s), lambda s: lc.cache_read(cache, at, outs, status=s)):
            outs = [torch.full((2, heads, dim), 4.0, device=DEV) for _ in range(2)]
            status = lc.alloc_status(DEV)
            fn(status)
            assert lc.last_status(status) == lc.ERR_INDEX
            fn(None)
            assert bool((outs[0] == 4.0).all()) and torch.equal(cache.codes, before[0]) and torch.equal(cache.scales, before[1])
    begin = torch.tensor([0, 10, 20], dtype=torch.int32, device=DEV)
    for table, first in (([[0, 8], [1, 2]], None), ([[0, -1], [1, 2]], None), ([[0, 1 << 30], [1, 2]], None), ([[0, 3], [1, 2]], [7, 0]), ([[0, 3], [1, 2]], [-1, 0]),
                         ([[0, 3], [1, 2]], [(1 << 31) - 1, 0])):
        status = lc.alloc_status(DEV)
        outs = [torch.full((20, heads, dim), 4.0, device=DEV) for _ in range(2)]
        lc.cache_read_pages(cache, torch.tensor(table, dtype=torch.int32, device=DEV), page, begin, outs,
                            None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV), status)
        assert lc.last_status(status) == lc.ERR_INDEX
        want = expected(k[8:], 8, 32)[2]  # the second sequence is whole
        assert torch.equal(outs[0][10:].cpu(), torch.cat([want[:8], want[8:10]]))
        untouched = (outs[0][:10] == 4.0).all(-1).all(-1)
        assert 0 < int(untouched.sum()) <= 10
    empty = lc.alloc_cache(0, heads, dim, 8, 32, DEV)
    status = lc.alloc_status(DEV)
    lc.cache_write(empty, k[:1], v[:1], torch.zeros(1, dtype=torch.int64, device=DEV), status)
    assert lc.last_status(status) == lc.ERR_INDEX


def test_nothing_to_do(lc):
    cache = lc.alloc_cache(8, 2, 16, 4, 32, DEV)
    none = torch.empty(0, 2, 16, device=DEV)
    at = torch.empty(0, dtype=torch.int64, device=DEV)
    lc.cache_write(cache, none, none, at)
    assert [tuple(t.shape) for t in lc.cache_read(cache, at)] == [(0, 2, 16)] * 2
    outs = [torch.full((3, 2, 16), 2.0, device=DEV) for _ in range(2)]
    zeros = torch.zeros(1, dtype=torch.int32, device=DEV)
    lc.cache_read_pages(cache, torch.empty(0, 4, dtype=torch.int32, device=DEV), 4, zeros, outs)
    lc.cache_read_pages(cache, torch.empty(1, 0, dtype=torch.int32, device=DEV), 4, torch.zeros(2, dtype=torch.int32, device=DEV), outs)
    assert bool((outs[0] == 2.0).all())


@pytest.mark.parametrize("bits", [4, 8])
def test_a_cache_beyond_32_bits(lc, bits):
    # codes at byte offsets past 2^32, values past 2^32
    heads, dim = 8, 128
    slots = ((1 << 32) // (heads * dim * bits // 8)) + 1000
    cache = lc.Cache(torch.empty(2, slots, heads, dim * bits // 8, dtype=torch.uint8, device=DEV),
                     torch.empty(2, slots, heads, 1, dtype=torch.bfloat16, device=DEV), dim, bits, 128)
    at = torch.tensor([0, slots - 1, slots - 1000, slots // 2], device=DEV)
    k, v = rows_of(4, heads, dim, "bf16", 8), rows_of(4, heads, dim, "bf16", 9)
    lc.cache_write(cache, k, v, at)
    for x, y in zip((k, v), lc.cache_read(cache, at, dtype=torch.float32)):
        assert torch.equal(y.cpu(), expected(x, bits, 128)[2])
    page = 1000
    table = torch.tensor([[(slots - 1) // page]], dtype=torch.int32, device=DEV)
    outs = [torch.empty(1, heads, dim, device=DEV) for _ in range(2)]
    lc.cache_read_pages(cache, table, page, torch.tensor([0, 1], dtype=torch.int32, device=DEV), outs,
                        torch.tensor([(slots - 1) % page], dtype=torch.int32, device=DEV))
    assert torch.equal(outs[1].cpu(), expected(v, bits, 128)[2][1:2])


def test_on_another_stream_and_in_a_graph(lc):
    heads, dim, n = 4, 64, 11
    cache = lc.alloc_cache(50, heads, dim, 4, 64, DEV)
    k, v = rows_of(n, heads, dim, "fp16", 1), rows_of(n, heads, dim, "fp16", 2)
    at = torch.randperm(50, device=DEV)[:n]
    outs = [torch.zeros(n, heads, dim, dtype=torch.float16, device=DEV) for _ in range(2)]

    def steps():
        lc.cache_write(cache, k, v, at)
        lc.cache_read(cache, at, outs)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(outs[0].cpu(), expected(k, 4, 64)[2].half())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    k.copy_(v * 2), at.copy_(torch.randperm(50, device=DEV)[:n])
    graph.replay()
    assert torch.equal(outs[0].cpu(), expected(k, 4, 64)[2].half()) and torch.equal(outs[1].cpu(), expected(v, 4, 64)[2].half())


def test_the_binding_refuses(lc):
    cache = lc.alloc_cache(8, 2, 16, 4, 32, DEV)
    k = torch.randn(3, 2, 16, device=DEV)
    at = torch.arange(3, device=DEV)
    for call in (lambda: lc.cache_write(cache, k, None, at), lambda: lc.cache_write(cache, k, k.half(), at), lambda: lc.cache_write(cache, k[:, :1], k[:, :1], at),
                 lambda: lc.cache_write(cache, k, k, at.int()), lambda: lc.cache_write(cache, k, k, at[:2]), lambda: lc.cache_write(cache, k.cpu(), k.cpu(), at),
                 lambda: lc.cache_write(cache, k.transpose(1, 2), k.transpose(1, 2), at), lambda: lc.cache_read(cache, at, [k]),
                 lambda: lc.cache_read(cache, at, [k, k[:, :, :8]]), lambda: lc.cache_write(cache, k, k, at, torch.zeros(1, device=DEV)),
                 lambda: lc.Cache(cache.codes[:, 1:].contiguous(), cache.scales, 16, 4, 32), lambda: lc.Cache(cache.codes, cache.scales, 99, 4, 32),
                 lambda: lc.cache_read_pages(cache, at.view(1, 3), 2, at.int(), [k, k]),
                 lambda: lc.cache_read_pages(cache, at.int().view(1, 3), 2, at.int(), [k, k])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lc.alloc_cache(8, 2, 16, 5, 32, DEV), lambda: lc.alloc_cache(8, 2, 16, 4, 33, DEV),
                 lambda: lc.cache_read(cache, at, [k[:1].expand(3, 2, 16), k]),
                 lambda: lc.cache_read_pages(cache, at.int().view(1, 3), 0, at[:2].int(), [k, k])):
        with pytest.raises(lc.LCError):
            call()
