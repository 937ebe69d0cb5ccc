"""What the sums of lc_q4_matvec keep: a term counts by its own size, |scale code x|, whatever else the vector holds. A weight of code 0
takes nothing from the others, however large x is there; small vectors and all bits of an fp32 one count.

The bound is that of test_gpu_q4: |error| <= S * (17 * G / 16 * 2^-23 + (cols / G + 16) * 2^-24) + half a step of the output's type,
S = sum |scale code x|: products with a code of 0 are 0, so that a sum of 17 numbers loses the last of 24 bits of the largest that counts.
"""
import numpy as np
import pytest
import torch

import quant_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# vectors of a pass: one, two and four eights of columns (an fp32 vector takes three)
TOKENS = {"fp32": (1, 2, 5, 10), "bf16": (1, 8, 16, 32), "fp16": (1, 8, 16, 32)}
# what stands on the codes of 0: all below what makes a sum overflow
LARGE = {"fp32": (1e4, 2.0 ** 30, 2.0 ** 45, 2.0 ** 95), "bf16": (1e4, 2.0 ** 30, 2.0 ** 45, 2.0 ** 95), "fp16": (1e4, 6e4)}


@pytest.fixture(scope="module")
def lc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding

    binding.lib()
    return binding


def check(lc, w, x, group):
    """Products of float64 weights (on the CPU) with vectors on the GPU, in fp32, within the bound."""
    q4 = lc.q4_quantize(w.float().to(DEV), group)
    codes, scales = ref.quantize(w.float().double().numpy(), 4, group)
    v, xd = torch.from_numpy(ref.values(codes, scales, group)), x.double().cpu()
    got = lc.q4_matvec(q4, x, torch.empty(x.shape[0], w.shape[0], device=DEV)).double().cpu()
    want, size = xd @ v.T, xd.abs() @ v.abs().T
    bound = size * (17 * group / 16 * 2.0 ** -23 + (w.shape[1] / group + 16) * 2.0 ** -24) + want.abs() * 2.0 ** -24 + 2.0 ** -149
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound.clamp(min=1e-300)).max())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
def test_one_weight_beside_a_large_value_on_a_zero(lc, kind, group):
    for rows in (16, 40, 5000):
        w = torch.zeros(rows, 256, dtype=torch.float64)
        w[:, 3] = 7.0  # scale 1, code 7; all other codes are 0
        w[1::3, 3] = -5.0
        q4 = lc.q4_quantize(w.float().to(DEV), group)
        for tokens in TOKENS[kind]:
            for large in LARGE[kind]:
                x = torch.ones(tokens, 256, device=DEV, dtype=TYPES[kind])
                x[:, 5] = large
                x[:, 17] = -large
                x[:, 100] = large
                got = lc.q4_matvec(q4, x, torch.empty(tokens, rows, device=DEV)).cpu()
                codes, scales = ref.quantize(w.numpy(), 4, group)
                want = torch.from_numpy(ref.values(codes, scales, group))[:, 3].expand(tokens, rows)
                assert torch.equal(got.double(), want), (rows, tokens, large)  # every other term is 0


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
def test_large_values_on_columns_of_zeros(lc, kind, group):
    for rows, cols in ((70, 900), (3000, 520)):
        g = torch.Generator().manual_seed(rows + group)
        w = torch.randn(rows, cols, generator=g, dtype=torch.float64) * torch.exp(torch.randn(rows, 1, generator=g, dtype=torch.float64))
        zeros = torch.randperm(cols, generator=g)[: cols // 8]
        w[:, zeros] = 0.0
        for tokens in TOKENS[kind]:
            for large in LARGE[kind]:
                x = torch.randn(tokens, cols, generator=g)
                x[:, zeros] = large * (0.5 + 0.5 * torch.rand(tokens, len(zeros), generator=g))
                check(lc, w, x.to(TYPES[kind]).to(DEV), group)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("kind", list(TYPES))
def test_vectors_of_one_sign_and_outliers(lc, kind, group):
    for rows, cols in ((130, 1100), (2600, 384)):
        g = torch.Generator().manual_seed(group)
        w = torch.randn(rows, cols, generator=g, dtype=torch.float64)
        w[:, ::5] *= 1e-2  # mostly codes of 0
        for tokens in TOKENS[kind]:
            x = torch.rand(tokens, cols, generator=g)
            check(lc, w, x.to(TYPES[kind]).to(DEV), group)
            x[:, ::5] *= 3e4
            check(lc, w, x.to(TYPES[kind]).to(DEV), group)
            check(lc, w, (-x).to(TYPES[kind]).to(DEV), group)


def diagonal(n):
    w = torch.zeros(n, n, dtype=torch.float64)
    w.fill_diagonal_(7.0)
    return w


@pytest.mark.parametrize("group", [32, 64, 128])
def test_all_bits_of_an_fp32_vector_where_no_sum_overflows(lc, group):
    # magnitudes far apart in every group, all below 2^47; 7 x needs 27 bits: the parts' products are exact, their sum is rounded twice at most
    n = 256
    q4 = lc.q4_quantize(diagonal(n).float().to(DEV), group)
    r = np.random.RandomState(group)
    for tokens in (1, 2, 5, 10):
        x = (r.randint(1 << 23, 1 << 24, (tokens, n)) * 2.0 ** r.randint(-140, 23, (tokens, n)) * r.choice([-1, 1], (tokens, n))).astype(np.float32)
        got = lc.q4_matvec(q4, torch.from_numpy(x).to(DEV)).cpu().numpy().astype(np.float64)
        want = 7.0 * x.astype(np.float64)
        assert np.all(np.abs(got - want) <= 2.0 ** -23 * np.abs(want))


@pytest.mark.parametrize("kind", list(TYPES))
def test_the_smallest_vectors_count(lc, kind):
    # multiples of the smallest number of the type; 7 times one is a whole number of fp32's smallest: exact. With scales of 2^60 too.
    n, step, most = 256, {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}[kind], {"fp32": 1 << 20, "bf16": 128, "fp16": 1024}[kind]
    r = np.random.RandomState(3)
    for scale in (1.0, 2.0 ** 60, 2.0 ** 100):
        q4 = lc.q4_quantize((diagonal(n) * scale).float().to(DEV), 64)
        for tokens in TOKENS[kind]:
            x = r.randint(-most, most + 1, (tokens, n)) * step
            xs = torch.from_numpy(x).to(TYPES[kind]).to(DEV)
            assert np.array_equal(xs.double().cpu().numpy(), x)
            got = lc.q4_matvec(q4, xs, torch.empty(tokens, n, device=DEV)).double().cpu().numpy()
            assert np.array_equal(got, 7.0 * scale * x)
