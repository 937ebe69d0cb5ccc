"""Attention to a quantised cache on the GPU, as close to the formula as its roundings allow (attend_bounds): every output, and the mean square of a batch. The inputs are such
that keys on both sides of a mask's borders weigh much, so that a mistake of one key shows (tests/test_attend_bounds.py tries that on the bounds)."""
import pytest
import torch

import attend_bounds as bounds
from test_gpu_attend import DEV, TYPES, Case, lc, values  # noqa: F401 (lc is a fixture)

pytestmark = pytest.mark.gpu


class Close(Case):
    def __init__(self, lc, kind, bits, group, heads, shared, dim, page, firsts, counts, seed=0):  # noqa: F811
        super().__init__(lc, kind, bits, group, heads, shared, dim, page, firsts, counts, seed=seed)
        g = torch.Generator(device=DEV).manual_seed(seed + 11)
        shape = (2, self.cache.slots, heads, dim)
        kv = torch.randn(shape, generator=g, device=DEV) * torch.exp(0.3 * torch.randn(shape[:3] + (1,), generator=g, device=DEV))
        lc.cache_write(self.cache, kv[0], kv[1], torch.arange(self.cache.slots, device=DEV))
        self.scale = 2.0 / dim ** 0.5
        held = values(self.cache)
        for s, n in enumerate(counts):
            if n:
                mine = slice(int(self.begin[s]), int(self.begin[s]) + n)
                self.q[mine] = bounds.telling(self.q[mine].double(), held[0][self.places(s)], firsts[s] + torch.arange(n, device=DEV)).to(self.kind)

    def places(self, s):
        at = torch.arange(self.firsts[s] + self.counts[s], device=DEV)
        return self.table[s].long()[at // self.page] * self.page + at % self.page

    def call(self, lc, **kw):  # noqa: F811
        return super().call(lc, scale=self.scale, **kw)

    def check(self, lc, got, mean=True, apart=False, prefix=None, **kw):  # noqa: F811
        held, cache = values(self.cache), self.cache
        off2, allowed2 = 0.0, 0.0
        for s, (first, n) in enumerate(zip(self.firsts, self.counts)):
            if n == 0:
                continue
            mine, place, shared = slice(int(self.begin[s]), int(self.begin[s]) + n), self.places(s), self.q.shape[1] // cache.heads
            many = self.kind != torch.float32 and cache.dim <= 128 and n > 16 // shared
            out, allowed, square = bounds.attend(self.kind, cache.bits, many, self.q[mine].double(), held[0][place], held[1][place], first + torch.arange(n, device=DEV), self.scale,
                                                 prefix=0 if prefix is None else int(prefix[s]), apart=apart, **kw)
            off = (got[mine].double() - out).abs()
            if self.kind == torch.float16:  # what is beyond the type's numbers may be Inf
                off = torch.where(out.abs() + allowed < 65504.0, off, 0.0)
            off = torch.where(allowed.isinf(), 0.0, off)
            assert bool((off <= allowed).all()), (s, float((off / allowed).max()), int((off > allowed).sum()), off.numel())
            off2, allowed2 = off2 + float((off ** 2).sum()), allowed2 + float(square.sum())
        assert lc.last_status(self.status) == lc.OK
        assert not mean or off2 <= allowed2, off2 / allowed2


BATCHES = {"tokens": ([3000, 900, 20000, 60, 0], [1, 1, 1, 1, 1]), "drafts": ([2000, 500, 70], [3, 2, 4]), "chunks": ([1500, 90, 0], [130, 64, 200]), "mixed": ([700, 4000, 33], [90, 1, 1])}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("bits,group", [(4, 32), (4, 128), (8, 64), (8, 128)])
@pytest.mark.parametrize("shared,dim", [(4, 64), (2, 80), (4, 128), (2, 256)])
@pytest.mark.parametrize("batch", list(BATCHES))
def test_close(lc, kind, bits, group, shared, dim, batch):  # noqa: F811
    case = Close(lc, kind, bits, group, 2, shared, dim, 16, *BATCHES[batch], seed=dim + bits)
    case.check(lc, case.call(lc))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("batch", ["tokens", "drafts", "chunks", "mixed"])
@pytest.mark.parametrize("options", ["cap 50", "cap 100", "slopes", "window", "prefix window", "scale below 0"])
def test_close_with_options(lc, kind, batch, options):  # noqa: F811
    case = Close(lc, kind, 8, 64, 2, 4, 128, 16, *BATCHES[batch], seed=len(options))
    kw = {}
    if "cap" in options:
        kw["cap"] = float(options.split()[1])
    if options == "slopes":
        kw["slopes"] = torch.tensor([0.05, 0.01, 0.002, 0.0, 0.1, 0.03, 0.0005, 0.2], device=DEV)
    if "window" in options:
        kw["window"] = 50
    if "prefix" in options:
        kw["prefix"] = torch.full((len(case.counts),), 45, dtype=torch.int32, device=DEV)
    if "below" in options:
        case.scale = -case.scale
    case.check(lc, case.call(lc, **kw), **kw)
