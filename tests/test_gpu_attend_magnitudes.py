"""Values near both ends of fp32's range, and scores so large that one key has it all."""
import pytest
import torch

from test_gpu_attend import DEV, TYPES, lc, values  # noqa: F401 (lc is a fixture)
from test_gpu_attend_close import Close

pytestmark = pytest.mark.gpu

BATCHES = {"tokens": ([3000, 9000, 60], [1, 1, 1]), "drafts": ([2000, 500], [3, 2]), "chunks": ([9000, 90], [130, 300]), "short": ([400], [1])}


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("power", [-100, -60, 60, 100, 115, 120])
@pytest.mark.parametrize("bits,dim", [(8, 128), (4, 64), (8, 256)])
@pytest.mark.parametrize("positive", [False, True])
def test_values_of_any_size(lc, kind, batch, power, bits, dim, positive):  # noqa: F811
    """Means of values stay in the range of the values, whatever the sums are."""
    case = Close(lc, kind, bits, 64, 2, 4, dim, 16, *BATCHES[batch], seed=dim)
    if positive:
        v = values(case.cache)[1].abs().float()
        keys = values(case.cache)[0].float()
        lc.cache_write(case.cache, keys, v, torch.arange(case.cache.slots, device=DEV))
    case.scale *= 0.25  # many keys weigh something
    case.cache.scales[1] = (case.cache.scales[1].float() * 2.0 ** power).to(torch.bfloat16)
    case.check(lc, case.call(lc))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("counts", [[1, 1], [3, 2], [40, 9]])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("scale", [1e5, 1e7, -1e9, 1e12, 1e20])
def test_the_largest_score_has_it_all(lc, kind, counts, dim, scale):  # noqa: F811
    """Where the largest score is ahead of the next by more than both may be off, the result is that key's values, rounded."""
    case = Close(lc, kind, 8, 64, 2, 4, dim, 16, [700, 60], counts, seed=dim)
    case.scale = scale
    got, held, told = case.call(lc), values(case.cache), 0
    for s, n in enumerate(counts):
        place = case.places(s)
        for h in range(8):
            mine = slice(int(case.begin[s]), int(case.begin[s]) + n)
            q, k, v = case.q[mine, h].double(), held[0][place, h // 4], held[1][place, h // 4]
            seen = torch.arange(place.numel(), device=DEV)[None, :] <= case.firsts[s] + torch.arange(n, device=DEV)[:, None]
            t = (scale * (q @ k.T)).masked_fill(~seen, -torch.inf)
            off = abs(scale) * (q.abs() @ k.abs().T).amax(-1) * 2.0 ** -9  # keys of 11 bits, twice
            top = t.topk(2, -1)
            clear = top.values[:, 0] - top.values[:, 1] > off + 200.0
            want = v[top.indices[:, 0]]
            step = 2.0 ** -8 if case.kind == torch.bfloat16 else 2.0 ** -10
            assert bool(((got[mine, h].double() - want).abs() <= 2 * step * want.abs() + 1e-7)[clear].all()), (s, h)
            told += int(clear.sum())
    assert told >= sum(counts)  # an eighth of them
    assert lc.last_status(case.status) == lc.OK


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("firsts,counts", [([60], [1]), ([300], [200]), ([9000], [130])])
def test_scores_that_are_all_minus_infinity(lc, kind, firsts, counts):  # noqa: F811
    """0 / 0 in the formula, and no number here, by either kernel, in blocks that one CTA has and in those that several share."""
    case = Close(lc, kind, 8, 64, 1, 4, 64, 16, firsts, counts, seed=1)
    ones = torch.ones(case.cache.slots, 1, 64, device=DEV)
    lc.cache_write(case.cache, ones, values(case.cache)[1].float(), torch.arange(case.cache.slots, device=DEV))
    case.cache.scales[0] *= 2.0 ** 100
    case.q.fill_(-1.0)
    case.scale = 1e25
    n = counts[0]
    assert bool(case.call(lc)[:n].isnan().all())
