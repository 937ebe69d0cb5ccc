"""Groups with the largest numbers of a type of 16 bits read back as numbers of it. Their scale may be rounded up, by 2^-8 at most, so
that code times scale lies beyond the type: such a value reads as the largest number, which is nearer to what was written."""
import numpy as np
import pytest
import torch

import quant_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def lc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding

    binding.lib()
    return binding


def rows_up_to_the_largest(kind, dim):
    """A row for each of the type's last 80 numbers, as its largest magnitude."""
    info = torch.finfo(TYPES[kind])
    last = torch.tensor(info.max, dtype=TYPES[kind]).view(torch.int16).item()
    most = torch.arange(last - 79, last + 1, dtype=torch.int16).view(TYPES[kind])
    g = torch.Generator().manual_seed(dim)
    x = ((torch.rand(80, dim, generator=g, dtype=torch.float64) * 2 - 1) * most.double()[:, None]).to(TYPES[kind])
    x[:, 0], x[:, dim - 1] = most, -most
    return x.to(DEV)


def check(x, got, bits, group):
    """Finite, and the nearest number to code times scale; beyond the type's largest number, that one."""
    codes, scales = ref.quantize(x.double().cpu().numpy(), bits, group)
    values, top = torch.from_numpy(ref.values(codes, scales, group)), torch.finfo(got.dtype).max
    assert bool(got.isfinite().all())
    assert torch.equal(got.cpu(), values.clamp(-top, top).to(torch.float32).to(got.dtype))
    step = torch.from_numpy(np.repeat(ref.bf16_values(scales), group, axis=-1)[:, : x.shape[1]])
    off, half = (got.double().cpu() - x.double().cpu()).abs(), torch.finfo(got.dtype).eps / 2
    assert bool((off <= step / 2 + values.abs() * half).all())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("dim", [128, 49])
def test_rows_of_a_cache(lc, kind, bits, dim):
    for group in (32, 64, 128):
        x = rows_up_to_the_largest(kind, dim)
        cache = lc.alloc_cache(96, 1, dim, bits, group, DEV, planes=1)
        at = torch.arange(80, device=DEV)
        lc.cache_write(cache, x.view(80, 1, dim), None, at)
        check(x, lc.cache_read(cache, at, dtype=TYPES[kind])[0].view(80, dim), bits, group)
        out = torch.empty(80, 1, dim, dtype=TYPES[kind], device=DEV)
        lc.cache_read_pages(cache, torch.arange(6, dtype=torch.int32, device=DEV).view(1, 6), 16, torch.tensor([0, 80], dtype=torch.int32, device=DEV), [out])
        check(x, out.view(80, dim), bits, group)


@pytest.mark.parametrize("kind", list(TYPES))
def test_weights(lc, kind):
    for group in (32, 64, 128):
        x = rows_up_to_the_largest(kind, 300)
        check(x, lc.q4_read(lc.q4_quantize(x, group), dtype=TYPES[kind]), 4, group)


def test_what_a_narrower_type_cannot_hold_is_still_inf(lc):
    x = torch.full((3, 1, 64), 1e6, device=DEV)
    x[1], x[2, 0, 5] = -7e4, float("nan")
    cache = lc.alloc_cache(3, 1, 64, 8, 32, DEV, planes=1)
    at = torch.arange(3, device=DEV)
    lc.cache_write(cache, x, None, at)
    got = lc.cache_read(cache, at, dtype=torch.float16)[0].cpu()
    assert bool((got[0] == float("inf")).all()) and bool((got[1] == -float("inf")).all())
    assert bool(got[2, 0, :32].isnan().all()) and bool((got[2, 0, 32:] == float("inf")).all())


def test_beyond_the_largest_of_bf16(lc):
    x = torch.full((2, 1, 64), torch.finfo(torch.float32).max, device=DEV)
    x[1] = -x[1]
    for bits in (4, 8):
        cache = lc.alloc_cache(2, 1, 64, bits, 32, DEV, planes=1)
        at = torch.arange(2, device=DEV)
        lc.cache_write(cache, x, None, at)
        got, top = lc.cache_read(cache, at, dtype=torch.bfloat16)[0], torch.finfo(torch.bfloat16).max
        assert bool((got[0] == top).all()) and bool((got[1] == -top).all())
    got = lc.q4_read(lc.q4_quantize(x.view(2, 64), 32), dtype=torch.bfloat16)
    assert bool((got[0] == top).all()) and bool((got[1] == -top).all())
