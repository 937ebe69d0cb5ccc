"""Capped scores on the GPU: a cap costs a score 2^-20 of itself, however large the cap is; in 16 bits, of caps up to 64, 2^-16 at most."""
import pytest
import torch

import attend_reference as ref
from test_gpu_attend import DEV, TYPES, Case, lc, values  # noqa: F401 (lc is a fixture)

pytestmark = pytest.mark.gpu


def check(lc, case, got, cap, slopes=None):  # noqa: F811
    """Like Case.check, with a bound that does not grow with the cap: that of scores without one, and 2^-20 of every score (at most the sum of its products), and 2^-16
    (see above), so twice that of the mean of |v|."""
    held = values(case.cache)
    for s, (first, n) in enumerate(zip(case.firsts, case.counts)):
        at = torch.arange(first + n, device=DEV)
        place = case.table[s].long()[at // case.page] * case.page + at % case.page
        mine = slice(int(case.begin[s]), int(case.begin[s]) + n)
        parts = ref.attend(case.q[mine].double(), held[0][place], held[1][place], first + torch.arange(n, device=DEV), case.scale, cap, slopes)
        off = (got[mine].double() - parts[0]).abs()
        d = 2.0 ** -20 * parts[2] + (2.0 ** -16 if cap <= 64 and case.kind != torch.float32 else 0.0)
        allowed = ref.bound(case.kind, *parts, case.cache.dim) + 2 * torch.expm1(d)[..., None] * parts[1]
        assert bool((off <= allowed).all()), (s, float((off / allowed).max()), float(off.max()))
    assert lc.last_status(case.status) == lc.OK


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("counts", [[1, 1], [6, 2], [150, 70]])
@pytest.mark.parametrize("cap", [0.5, 8.0, 30.0, 1e3, 1e4, 1e6, 1e8, 1e30])
@pytest.mark.parametrize("slopes", [False, True])
def test_caps_of_every_size(lc, kind, counts, cap, slopes):  # noqa: F811
    case = Case(lc, kind, 8, 64, 2, 2, 64, 16, [300, 40], counts, seed=3, spread=0.3)
    kw = {"slopes": torch.tensor([0.01, 0.2, 0.0, 0.05], device=DEV)} if slopes else {}
    check(lc, case, case.call(lc, cap=cap, **kw), cap, **kw)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("counts", [[1], [150]])
def test_a_cap_beyond_all_scores_is_none(lc, kind, counts):  # noqa: F811
    """Scores hundreds of thousands of times smaller than the cap are what they are without it, to some roundings of fp32: weights are off by 2^-20 of the scores at
    most, and results then at most by that much and a rounding each."""
    case = Case(lc, kind, 8, 64, 2, 2, 64, 16, [300], counts, seed=4, spread=0.3)
    plain, capped = case.call(lc), case.call(lc, cap=1e9)
    size = float(plain[: counts[0]].float().abs().max())
    step = 2 * ref.HALF_STEP[case.kind]
    assert float((plain - capped).float().abs().max()) <= (2 * step + 2.0 ** -14) * size
