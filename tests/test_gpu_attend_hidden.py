"""Keys and values that a row does not see, however large they are, take nothing from those that it sees."""
import pytest
import torch

from test_gpu_attend import DEV, lc  # noqa: F401 (lc is a fixture)
from test_gpu_attend_close import Close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("bits,dim", [(4, 64), (8, 128), (8, 80)])
@pytest.mark.parametrize("planes", ["keys", "values", "both"])
@pytest.mark.parametrize("power", [9, 13, 16, 20, 30, 60])
@pytest.mark.parametrize("counts", [[150, 40, 7], [300, 1, 90]])
@pytest.mark.parametrize("kw", [{}, {"window": 60}])
def test_large_ones_behind_a_row_or_ahead_of_its_window(lc, kind, bits, dim, planes, power, counts, kw):  # noqa: F811
    """Some keys of each sequence are 2^power times as large as the others: one in the middle of the new rows, one at their end, one some way ahead of them. Rows that see none of
    them are held to what they are without, rows that do to what their own largest ones allow."""
    case = Close(lc, kind, bits, 32, 2, 4, dim, 16, [200, 900, 33], counts, seed=power)
    for s, n in enumerate(counts):
        place = case.places(s)
        at = {case.firsts[s] + n // 2, case.firsts[s] + n - 1} | ({case.firsts[s] - 20} if kw else set())
        for p in at:
            for plane in {"keys": [0], "values": [1], "both": [0, 1]}[planes]:
                case.cache.scales[plane, place[p]] *= 2.0 ** power
    case.check(lc, case.call(lc, **kw), mean=False, apart=True, **kw)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("window", [0, 100])
def test_sizes_that_change_from_key_to_key(lc, kind, window):  # noqa: F811
    """Values over 40 binades, in every order: rising, falling, at random; the largest is seen by some rows or by all."""
    for order in ("rising", "falling", "random"):
        case = Close(lc, kind, 8, 64, 2, 4, 128, 16, [300, 0], [200, 120], seed=3)
        for s in range(2):
            place = case.places(s)
            n = place.numel()
            powers = torch.linspace(-20, 20, n, device=DEV).round()
            powers = powers.flip(0) if order == "falling" else powers[torch.randperm(n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(s))] if order == "random" else powers
            case.cache.scales[1, place] = (case.cache.scales[1, place].float() * torch.exp2(powers)[:, None, None]).to(torch.bfloat16)
        kw = {"window": window} if window else {}
        case.check(lc, case.call(lc, **kw), mean=False, apart=True, **kw)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("options", ["cap 30", "cap 1000", "slopes", "prefix window", "scale below 0", "none"])
def test_with_options_and_parts_of_several_ctas(lc, kind, options):  # noqa: F811
    """Long sequences, whose blocks several CTAs share, with some values 2^18 times as large as the others and some keys 2^-18 times, ahead of tiles without such and behind."""
    case = Close(lc, kind, 8, 32, 2, 4, 128, 64, [9000, 0, 500], [70, 700, 300], seed=len(options))
    for s in range(3):
        place = case.places(s)
        n = place.numel()
        some = torch.arange(n // 3, n // 2, 7, device=DEV)
        case.cache.scales[1, place[some]] *= 2.0 ** 18
        case.cache.scales[0, place[some + 1]] *= 2.0 ** -18
    kw = {}
    if "cap" in options:
        kw["cap"] = float(options.split()[1])
    if options == "slopes":
        kw["slopes"] = torch.tensor([0.05, 0.01, 0.002, 0.0, 0.1, 0.03, 0.0005, 0.2], device=DEV)
    if "window" in options:
        kw["window"], kw["prefix"] = 50, torch.full((3,), 45, dtype=torch.int32, device=DEV)
    if "below" in options:
        case.scale = -case.scale
    got = case.call(lc, **kw)
    case.check(lc, got, mean=False, apart=True, **kw)
    assert torch.equal(got, case.call(lc, **kw))


def test_zeros_ahead_of_the_first_values(lc):  # noqa: F811
    case = Close(lc, "bf16", 8, 64, 2, 4, 64, 16, [300, 0], [40, 200], seed=5)
    for s in range(2):
        case.cache.scales[1, case.places(s)[:130]] = 0.0
        case.cache.scales[0, case.places(s)[100:150]] = 0.0
    case.check(lc, case.call(lc), mean=False)
