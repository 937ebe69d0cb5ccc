"""What the Python calls on a cache's pages refuse ahead of the library, without a GPU: tensors that say they are on a device, and a library that must not be reached."""
import pytest
import torch

from paper_2009_13003_b200 import binding


class OnDevice(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 0


def on(t):
    return torch.Tensor._make_subclass(OnDevice, t)


@pytest.fixture
def reached(monkeypatch):
    calls = []
    monkeypatch.setattr(binding, "_call", lambda name, *args: calls.append(name))
    return calls


def attend(**kw):
    shape = binding.LCCache(None, None, 32, 2, 1, 64, 8, 64)
    codes = on(torch.zeros(2, 32, 1, binding.lib().lc_cache_code_bytes(shape) // 64, dtype=torch.uint8))
    cache = binding.Cache(codes, on(torch.zeros(2, 32, 1, 1, dtype=torch.bfloat16)), 64, 8, 64)
    size = int(binding.lib().lc_cache_attend_bytes(cache._c, 1))
    ints = lambda *x: on(torch.tensor(x, dtype=torch.int32))
    args = dict(dict(cache=cache, q=on(torch.zeros(2, 4, 64)), table=on(torch.zeros(1, 2, dtype=torch.int32)), page=16, begin=ints(0, 2), out=on(torch.zeros(2, 4, 64)),
                     workspace=on(torch.zeros(size, dtype=torch.uint8))), **kw)
    return binding.cache_attend(**args), size


def test_a_workspace_has_its_bytes_one_behind_the_other(reached):
    _, size = attend()
    assert reached == ["lc_cache_attend"]
    # as many elements, but one byte of memory; every second byte
    for bad in (on(torch.zeros(1, dtype=torch.uint8).expand(size)), on(torch.zeros(2 * size, dtype=torch.uint8)[::2]), on(torch.zeros(size, dtype=torch.int8))):
        with pytest.raises(ValueError):
            attend(workspace=bad)
    assert reached == ["lc_cache_attend"]


@pytest.mark.parametrize("page", [-1, (1 << 32) + 16, 1 << 32])
def test_a_page_that_does_not_fit_into_32_bits_is_not_another_one(reached, page):
    ints = lambda *shape: on(torch.zeros(shape, dtype=torch.int32))
    with pytest.raises(binding.LCError):
        binding.Pages(ints(3, 4), ints(3), ints(12), ints(1), page)
    with pytest.raises(binding.LCError):
        attend(page=page)
    codes = on(torch.zeros(1, 32, 1, 64, dtype=torch.uint8))
    cache = binding.Cache(codes, on(torch.zeros(1, 32, 1, 1, dtype=torch.bfloat16)), 64, 8, 64)
    with pytest.raises(binding.LCError):
        binding.cache_read_pages(cache, ints(1, 2), page, ints(2), [on(torch.zeros(2, 1, 64))])
    assert reached == []
