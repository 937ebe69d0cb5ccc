"""Values of the cache that are no numbers, among many rows and keys: they reach the rows that see them, in their group, and cost nobody else a bit or much time."""
import numpy as np
import pytest
import torch

from test_gpu_attend import DEV, Case, lc  # noqa: F401 (lc is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kw", [{}, {"window": 70}, {"prefix": 300}])
def test_only_where_they_are_seen(lc, kind, group, kw):
    """Several sequences in one call, blocks of several tiles: every row is compared with what it may see."""
    case = Case(lc, kind, 8, group, 2, 2, 128, 16, [500, 0, 130], [300, 200, 170], seed=group, spread=0.5)
    if "prefix" in kw:
        kw = {"prefix": torch.full((3,), kw["prefix"], dtype=torch.int32, device=DEV), "window": 40}
    clean = case.call(lc, **kw)
    groups = 128 // group
    bad = [(0, 3, 0, 0), (0, 499, 1, groups - 1), (0, 640, 0, 0), (2, 0, 0, groups - 1), (2, 299, 1, 0)]  # sequence, position, head of the cache, group
    for n, (s, p, h, g) in enumerate(bad):
        place = int(case.table[s, p // 16]) * 16 + p % 16
        case.cache.scales[1, place, h, g] = float("nan") if n % 2 else float("inf")
    got = case.call(lc, **kw)
    assert lc.last_status(case.status) == lc.OK
    broken = torch.zeros(got.shape, dtype=torch.bool, device=DEV)
    for s, p, h, g in bad:
        lo, n = int(case.begin[s]), case.counts[s]
        at = case.firsts[s] + torch.arange(n, device=DEV)
        seen = (at >= p) & (at - p < kw.get("window", 1 << 30))
        if "prefix" in kw:
            seen |= p < int(kw["prefix"][s])
        broken[lo : lo + n, 2 * h : 2 * h + 2, group * g : group * (g + 1)] |= seen[:, None, None]
    assert bool(got[broken].isnan().all())
    assert torch.equal(got[~broken], clean[~broken])


def test_behind_millions_of_keys(lc):
    """No warp waits longer for the others than it does without them."""
    length, rows, shared = 4 << 20, 2400, 16
    cache = lc.alloc_cache(length + 4096, 1, 64, 4, 64, DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    cache.codes.copy_(torch.randint(0, 255, cache.codes.shape, dtype=torch.uint8, generator=g, device=DEV))
    cache.scales.copy_((0.1 + torch.rand(cache.scales.shape, generator=g, device=DEV)).to(cache.scales.dtype))
    cache.scales[1, :: 100_000] = float("nan")
    table = torch.randperm((length + 4096) // 64, generator=g, device=DEV).to(torch.int32)[None]
    q = torch.randn(rows, shared, 64, generator=g, device=DEV).to(torch.bfloat16)
    status = lc.alloc_status(DEV)
    begin, first = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, rows], [length - rows]))
    out = lc.cache_attend(cache, q, table, 64, begin, first=first, status=status)
    assert lc.last_status(status) == lc.OK
    assert bool(out.isnan().all())
