"""Plans and attention without a GPU: the reference against a second reading of the text, sizes, and what the entry points refuse (made-up addresses: the checks
come before anything is touched)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import attend_reference as ref
from paper_2009_13003_b200 import binding


def test_the_reference_is_the_formula():
    g = torch.Generator().manual_seed(1)
    q, k, v = torch.randn(4, 6, 8, generator=g).double(), torch.randn(9, 2, 8, generator=g).double(), torch.randn(9, 2, 8, generator=g).double()
    slopes = torch.tensor([0.1, 0.2, 0.0, 0.5, 1.0, 0.3])
    positions = torch.tensor([3, 4, 5, 8])
    out = ref.attend(q, k, v, positions, 0.4, cap=1.5, slopes=slopes, window=3, prefix=2)[0]
    for r in range(4):
        for h in range(6):
            top, total = torch.zeros(8, dtype=torch.float64), 0.0
            for p in range(9):
                i = int(positions[r])
                if not (p < 2 or i - 3 < p <= i):
                    continue
                t = 1.5 * math.tanh(0.4 * float(q[r, h] @ k[p, h // 3]) / 1.5) - float(slopes[h]) * abs(i - p)
                top += math.exp(t) * v[p, h // 3]
                total += math.exp(t)
            assert torch.allclose(out[r, h], top / total, rtol=1e-12, atol=0)


def test_the_plan_of_the_reference():
    table, held, spare = np.array([[5, 6, -1], [7, -1, -1], [1, 2, 3]], np.int32), [5, 4, 12], np.array([8, 0, 4, -1, -1, -1, -1, -1], np.int32)
    begin, first, slots, after, count, table, spare = ref.plan(table, held, spare, 3, [4, 1, -1], 4, 6)
    # sequence 2 gives back 1, 2, 3; sequence 0 takes 3 for position 8, sequence 1 takes 2 for position 4
    assert begin == [0, 4, 5, 5] and first == [5, 4, 0] and after == [9, 5, 0] and count == 4
    assert slots == [25, 26, 27, 12, 8, -1] and spare.tolist() == [8, 0, 4, 1, 2, 3, -1, -1] and table[:2].tolist() == [[5, 6, 3], [7, 2, -1]]


def cache(**kw):
    d = dict(dict(codes=0x10000, scales=0x20000, slots=64, planes=2, heads=2, dim=64, bits=8, group=64), **kw)
    return binding.LCCache(*[d[k] for k in ("codes", "scales", "slots", "planes", "heads", "dim", "bits", "group")])


def test_sizes():
    L = binding.lib()
    size = L.lc_cache_attend_bytes(cache(), 3)
    assert size > 0 and size % 256 == 0 and size == L.lc_cache_attend_bytes(cache(slots=0), 3) == L.lc_cache_attend_bytes(cache(heads=8, dim=256, bits=4), 3)
    assert L.lc_cache_attend_bytes(cache(), 1 << 20) > size
    for bad in (dict(planes=1), dict(dim=257), dict(bits=5), dict(group=48), dict(heads=0)):
        assert L.lc_cache_attend_bytes(cache(**bad), 3) == 0, bad
    assert L.lc_cache_attend_bytes(None, 3) == 0 and L.lc_cache_attend_bytes(cache(), 1 << 31) == 0


def test_attend_refuses():
    L, A = binding.lib(), binding.ERR_ARG
    size = L.lc_cache_attend_bytes(cache(), 3)

    def call(c=None, kind=1, rows=5, q=(0x30000, 256, 64), out=(0x40000, 256, 64), ws=0x50000, wsize=size, status=None, null=(), **kw):
        d = dict(dict(table=0x60000, table_stride=4, width=4, page=16, begin=0x70000, first=0x80000, sequences=3, longest=0, heads=4, window=0, scale=0.1, cap=0.0, slopes=None,
                      prefix=None), **kw)
        how = binding.LCAttend(*[d[k] for k, _ in binding.LCAttend._fields_])
        refs = dict(cache=C.byref(c or cache()), q=C.byref(binding.LCRows(*q)), out=C.byref(binding.LCRows(*out)), how=C.byref(how))
        refs.update({k: None for k in null})
        return L.lc_cache_attend(refs["cache"], refs["q"], refs["out"], kind, rows, refs["how"], ws, wsize, status, None)

    for bad in (dict(null=("cache",)), dict(null=("q",)), dict(null=("out",)), dict(null=("how",)), dict(kind=3), dict(kind=-1), dict(c=cache(planes=1)), dict(c=cache(dim=300)),
                dict(c=cache(bits=3)), dict(c=cache(codes=None)), dict(c=cache(codes=0x10008)), dict(c=cache(scales=0x20002)), dict(heads=3), dict(heads=0), dict(heads=1 << 17),
                dict(rows=1 << 31), dict(rows=1 << 28), dict(page=0), dict(page=1 << 31), dict(sequences=1 << 31), dict(table_stride=3), dict(table_stride=1 << 32), dict(window=1 << 31),
                dict(scale=math.nan), dict(scale=math.inf), dict(scale=2e30), dict(cap=-0.5), dict(cap=math.nan), dict(cap=math.inf), dict(table=None), dict(table=0x60002),
                dict(begin=None), dict(begin=0x70001), dict(first=0x80002), dict(prefix=0x80002), dict(slopes=0x80002), dict(status=0x90002), dict(ws=None), dict(ws=0x50010),
                dict(q=(None, 256, 64)), dict(q=(0x30001, 256, 64)), dict(q=(0x30000, 1 << 33, 64)), dict(out=(0x40000, 255, 64)), dict(out=(0x40000, 256, 63)),
                dict(out=(0x40000, 64, 300)), dict(out=(0x40000, 0, 64)), dict(kind=0, q=(0x30002, 256, 64))):
        assert call(**bad) == A, bad
    assert call(wsize=size - 256) == binding.ERR_CAPACITY
    assert call(rows=0) == call(sequences=0) == binding.OK  # nothing to do


def test_plan_refuses():
    L, A = binding.lib(), binding.ERR_ARG

    def call(null=(), sequences=3, rows=8, tokens=0x10000, begin=0x20000, first=0x30000, slots=0x40000, held_after=0x50000, count_after=0x60000, status=None, **kw):
        d = dict(dict(table=0x70000, table_stride=4, held=0x80000, spare=0x90000, count=0xA0000, width=4, page=16, pages=12), **kw)
        books = binding.LCPages(*[d[k] for k, _ in binding.LCPages._fields_])
        return L.lc_cache_plan(None if null else C.byref(books), tokens, sequences, rows, begin, first, slots, held_after, count_after, status, None)

    for bad in (dict(null=True), dict(page=0), dict(page=1 << 31), dict(pages=1 << 31), dict(sequences=1 << 31), dict(rows=1 << 31), dict(table_stride=3), dict(table_stride=1 << 32),
                dict(table=None), dict(held=None), dict(spare=None), dict(count=None), dict(tokens=None), dict(begin=None), dict(first=None), dict(slots=None), dict(held_after=None),
                dict(count_after=None), dict(table=0x70002), dict(held=0x80001), dict(spare=0x90002), dict(count=0xA0002), dict(tokens=0x10002), dict(begin=0x20002), dict(first=0x30002),
                dict(slots=0x40004), dict(held_after=0x50002), dict(count_after=0x60002), dict(status=0x10001)):
        assert call(**bad) == A, bad
