"""Values of 16 bits through the quantisers: every code at every border, and the largest numbers of a type."""
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


def every_magnitude(kind, lo, hi):
    """All numbers of the type from lo to hi, as float64."""
    v = torch.arange(0, 0x7C00 if kind == "fp16" else 0x7F80, dtype=torch.int32).to(torch.int16).view(TYPES[kind]).double().numpy()
    return v[(v >= lo) & (v <= hi)]


def groups_of_all_codes(kind, bits, most):
    """Rows of 32: `most` ahead of each, behind it all smaller numbers that a code of 0 ... Q can come from, signs in turn."""
    top = 2 ** (bits - 1) - 1
    x = every_magnitude(kind, most / top / 4, most)
    x = x * np.where(np.arange(x.size) % 2, -1.0, 1.0)
    x = np.pad(x, (0, -x.size % 31)).reshape(-1, 31)
    return np.concatenate([np.full((x.shape[0], 1), most), x], axis=1)


# the largest magnitude's binade: scales from the smallest one on, one in the middle, the largest
BINADES = {"bf16": {4: [-124, -123, -122, -121, -118, -110, -100, 0, 127], 8: [-120, -119, -118, -117, -114, -106, 0, 127]},
           "fp16": {4: [-24, -20, -14, 0, 15], 8: [-24, -20, -14, 0, 15]}}


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("kind", list(TYPES))
def test_every_value_at_every_scale(lc, kind, bits):
    for binade in BINADES[kind][bits]:
        mosts = every_magnitude(kind, 2.0 ** binade, 2.0 ** (binade + 1) * (1 - 2.0 ** -12))
        mosts = mosts[:: 8 if kind == "fp16" and bits == 8 else 1]
        x = np.concatenate([groups_of_all_codes(kind, bits, m) for m in mosts])
        t = torch.from_numpy(x).to(TYPES[kind]).to(DEV)
        assert np.array_equal(t.double().cpu().numpy(), x)
        codes, scales = ref.quantize(x, bits, 32)
        n = x.shape[0]
        # whole rows of the cache, and rows off 16 bytes
        wide = torch.zeros(n, 1, 33, dtype=TYPES[kind], device=DEV)
        wide[:, 0, 1:] = t
        for rows in (t.view(n, 1, 32), wide[:, :, 1:]):
            cache = lc.alloc_cache(n, 1, 32, bits, 32, DEV, planes=1)
            lc.cache_write(cache, rows, None, torch.arange(n, device=DEV))
            assert np.array_equal(cache.scales[0].view(torch.int16).cpu().numpy().view(np.uint16).reshape(n, 1), scales)
            got = ref.cache_unpack(cache.codes[0].cpu().numpy().reshape(n, -1), 32, bits)
            wrong = got != codes
            assert not wrong.any(), (binade, int(wrong.sum()), x[wrong][:4], got[wrong][:4], codes[wrong][:4])
        if bits == 4:
            got, got_scales = ref.q4_unpack(lc.q4_quantize(t, 32).data.cpu().numpy(), n, 32, 32)
            assert np.array_equal(got[:n, :32], codes) and np.array_equal(got_scales[:n, :1], scales)
