"""State in few bits, without a GPU: the reference against exact fractions, sizes against the text, and what the entry points refuse
(made-up addresses: the checks come before anything is touched)."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

import quant_reference as ref
from paper_2009_13003_b200 import binding


def nearest(q):
    """The whole number nearest to a fraction, ties to even."""
    low = q.numerator // q.denominator
    rest = q - low
    return low + (1 if rest > Fraction(1, 2) or (rest == Fraction(1, 2) and low % 2) else 0)


def scale_of(most, top):
    q = Fraction(float(most)) / top
    if q == 0:
        return Fraction(0)
    unit = Fraction(1)
    while q / unit >= 256:
        unit *= 2
    while q / unit < 128:
        unit /= 2
    unit = max(unit, Fraction(1, 2**133))
    s = nearest(q / unit) * unit
    return s if s >= Fraction(1, 2**126) else Fraction(0)


@pytest.mark.parametrize("bits", [4, 8])
def test_the_reference_is_the_text(bits):
    r = np.random.RandomState(bits)
    top = 2 ** (bits - 1) - 1
    rows = [r.randn(70).astype(np.float32) * np.float32(10.0 ** k) for k in (-37, -30, -3, 0, 5, 30)]
    rows.append(np.zeros(70, np.float32))
    rows.append((np.arange(70) % (2 * top + 1) - top).astype(np.float32) / 2)  # on borders wherever the code is odd
    rows.append(np.float32(2.0 ** -126) * r.randint(-2 * top, 2 * top, 70).astype(np.float32) / 2)
    x = np.stack(rows).astype(np.float64)
    codes, scales = ref.quantize(x, bits, 32)
    for i in range(x.shape[0]):
        for g in range(3):
            part = x[i, 32 * g : 32 * g + 32]
            s = scale_of(np.abs(part).max(), top)
            assert Fraction(float(ref.bf16_values(scales[i, g]))) == s
            for j, w in enumerate(part):
                want = nearest(Fraction(float(w)) / s) if s else 0
                assert codes[i, 32 * g + j] == want and abs(want) <= top


def test_sizes_are_those_of_the_text():
    L = binding.lib()
    for rows, cols, group in [(1, 1, 32), (16, 128, 128), (17, 129, 64), (4097, 5003, 32), (50257, 2048, 128)]:
        assert L.lc_q4_bytes(rows, cols, group) == ref.q4_bytes(rows, cols, group)
    assert L.lc_q4_bytes(0, 5, 32) == L.lc_q4_bytes(5, 0, 32) == 0
    assert L.lc_q4_bytes(16, 128, 48) == L.lc_q4_bytes(1 << 31, 1, 32) == L.lc_q4_bytes(1, (1 << 31) - 128, 32) == 0
    assert L.lc_q4_bytes(1 << 30, 1 << 20, 32) == 0  # more groups than the kernels count
    cache = lambda **kw: binding.LCCache(None, None, *[dict(dict(slots=10, planes=2, heads=3, dim=49, bits=4, group=32), **kw)[k]
                                                       for k in ("slots", "planes", "heads", "dim", "bits", "group")])
    assert L.lc_cache_code_bytes(cache()) == 2 * 10 * 3 * 7 * 4 and L.lc_cache_scale_bytes(cache()) == 2 * 10 * 3 * 2 * 2
    assert L.lc_cache_code_bytes(cache(bits=8, planes=1, dim=128)) == 10 * 3 * 128
    assert L.lc_cache_code_bytes(cache(slots=1 << 33)) == (1 << 33) * 2 * 3 * 28
    for bad in (dict(bits=5), dict(group=48), dict(planes=3), dict(planes=0), dict(heads=0), dict(dim=0), dict(dim=65537), dict(slots=1 << 40)):
        assert L.lc_cache_code_bytes(cache(**bad)) == L.lc_cache_scale_bytes(cache(**bad)) == 0
    assert L.lc_cache_code_bytes(None) == 0


def test_weights_refuse():
    L, A, CAP = binding.lib(), binding.ERR_ARG, binding.ERR_CAPACITY
    w, q4, ws, x, out = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000
    big = 1 << 20
    quant = lambda w=w, kind=0, rows=20, cols=200, stride=200, group=64, q4=q4, size=big, ws=ws, wsize=big: L.lc_q4_quantize(
        w, kind, rows, cols, stride, group, q4, size, ws, wsize, None)
    for bad in (dict(w=None), dict(w=w + 2), dict(kind=3), dict(kind=-1), dict(stride=199), dict(group=16), dict(q4=None), dict(q4=q4 + 16), dict(ws=None),
                dict(ws=ws + 16), dict(rows=1 << 31), dict(cols=1 << 31)):
        assert quant(**bad) == A, bad
    assert quant(size=ref.q4_bytes(20, 200, 64) - 1) == CAP and quant(wsize=16) == CAP
    read = lambda out=out, kind=0, stride=200, q4=q4, size=big: L.lc_q4_read(q4, size, 20, 200, 64, out, kind, stride, None)
    for bad in (dict(out=None), dict(out=out + 1), dict(kind=7), dict(stride=100), dict(q4=None)):
        assert read(**bad) == A, bad
    assert read(size=100) == CAP
    mul = lambda x=x, kind=1, tokens=3, xs=200, out=out, okind=1, os=20, size=big, group=64: L.lc_q4_matvec(
        q4, size, 20, 200, group, x, kind, tokens, xs, out, okind, os, None)
    for bad in (dict(x=None), dict(x=x + 1), dict(kind=9), dict(okind=2), dict(okind=9), dict(kind=0, okind=1), dict(xs=199), dict(xs=1), dict(os=19), dict(out=None),
                dict(out=out + 1), dict(group=1), dict(tokens=binding.Q4_MAX_TOKENS + 1)):
        assert mul(**bad) == A, bad
    assert mul(size=64) == CAP
    assert mul(tokens=0) == binding.OK  # nothing to do
    assert L.lc_q4_matvec(None, 0, 0, 200, 64, x, 1, 3, 200, out, 1, 20, None) == binding.OK
    rec = lambda rows=20, cols=200, scratch=0x60000, base=w: L.lc_recover_q4(base, None, None, 1, rows, cols, 64, q4, big, scratch, ws, big, None)
    assert rec() == A and rec(rows=1 << 20, cols=1 << 13) in (A, CAP)


def test_the_cache_refuses():
    L, A = binding.lib(), binding.ERR_ARG
    slots = 0x70000

    def call(fn, n=5, kind=1, cache=None, planes=None, at=slots, status=None):
        c = binding.LCCache(*[dict(dict(codes=0x10000, scales=0x20000, slots=64, planes=2, heads=3, dim=40, bits=4, group=32), **(cache or {}))[k]
                              for k in ("codes", "scales", "slots", "planes", "heads", "dim", "bits", "group")])
        rows = (binding.LCRows * 2)(*(planes or [(0x30000, 120, 40), (0x40000, 120, 40)]))
        if fn == "pages":
            return L.lc_cache_read_pages(C.byref(c), rows, kind, n, 0x50000, 4, 4, 16, at, None, 2, status, None)
        return (L.lc_cache_write if fn == "write" else L.lc_cache_read)(C.byref(c), rows, kind, n, at, status, None)

    for fn in ("write", "read", "pages"):
        for bad in (dict(kind=3), dict(at=None), dict(at=slots + 2), dict(status=2), dict(n=1 << 31), dict(n=1 << 30), dict(cache=dict(codes=None)),
                    dict(cache=dict(codes=0x10004)), dict(cache=dict(scales=None)), dict(cache=dict(bits=3)), dict(cache=dict(group=0)), dict(cache=dict(heads=0)),
                    dict(planes=[(None, 120, 40), (0x40000, 120, 40)]), dict(planes=[(0x30000, 120, 40), (0x40001, 120, 40)]),
                    dict(planes=[(0x30000, 1 << 33, 40), (0x40000, 120, 40)])):
            assert call(fn, **bad) == A, (fn, bad)
        assert call(fn, n=0) == binding.OK
    # rows that are written must not share memory
    for strides in ((119, 40), (0, 40), (120, 39), (40, 40), (39, 200)):
        assert call("read", planes=[(0x30000, 120, 40), (0x40000,) + strides]) == A
    c = binding.LCCache(0x10000, 0x20000, 64, 2, 3, 40, 4, 32)
    rows = (binding.LCRows * 2)((0x30000, 120, 40), (0x40000, 120, 40))
    pages = lambda table=0x50000, stride=4, width=4, page=16, begin=0x60000, first=None, n=2: L.lc_cache_read_pages(
        C.byref(c), rows, 1, 5, table, stride, width, page, begin, first, n, None, None)
    for bad in (dict(table=None), dict(table=0x50002), dict(stride=3), dict(page=0), dict(page=1 << 31), dict(begin=None), dict(begin=0x60002), dict(first=2),
                dict(stride=1 << 32)):
        assert pages(**bad) == A, bad
    assert pages(n=0) == binding.OK


def test_the_words_for_a_bad_index():
    assert binding.lib().lc_strerror(binding.ERR_INDEX) == b"a slot or page that the cache does not have"


def test_sizes_of_a_cache_do_not_wrap():
    """A cache whose codes would take 2^62 bytes or more has no size and no call takes it: no small number left over from 2^64."""
    L = binding.lib()
    rows = (binding.LCRows * 2)((0x30000, 1 << 32, 1 << 16), (0x40000, 1 << 32, 1 << 16))
    for planes, heads, dim, bits, group in ((2, 65536, 32767, 8, 128), (2, 65536, 32767, 4, 32), (1, 1, 65536, 8, 32), (2, 65536, 1, 4, 128), (2, 32768, 65535, 8, 64)):
        for slots in (1 << 20, 1 << 30, 1 << 31, 1 << 32, 1 << 33, 1 << 36, (1 << 40) - 1):
            c = binding.LCCache(0x10000, 0x20000, slots, planes, heads, dim, bits, group)
            size = planes * slots * heads * (-(-dim // 8) * bits)
            fits = size < 1 << 62
            assert L.lc_cache_code_bytes(C.byref(c)) == (size if fits else 0), (slots, heads, dim)
            assert L.lc_cache_scale_bytes(C.byref(c)) == (planes * slots * heads * -(-dim // group) * 2 if fits else 0), (slots, heads, dim)
            assert L.lc_cache_write(C.byref(c), rows, 1, 0, 0x70000, None, None) == (binding.OK if fits else binding.ERR_ARG)
