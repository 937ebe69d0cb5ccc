"""The vectors of one lc_q4_matvec do not touch each other: an Inf, a NaN or a value that makes a sum overflow changes no bit of what the
other vectors give."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# a row's vectors side by side: one, two and four eights of columns (an fp32 vector takes three), two passes
TOKENS = {"fp32": (2, 5, 10, 23), "bf16": (3, 8, 16, 32, 40), "fp16": (3, 8, 16, 32, 40)}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,group", [(40, 300, 32), (3000, 520, 64), (64, 9000, 128), (30, 4096, 128)])
def test_a_vector_that_overflows_leaves_the_others_alone(kind, rows, cols, group):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding as lc

    g = torch.Generator(device=DEV).manual_seed(rows)
    q4 = lc.q4_quantize(torch.randn(rows, cols, generator=g, device=DEV), group)
    big = torch.finfo(TYPES[kind]).max
    for tokens in TOKENS[kind]:
        x = torch.randn(tokens, cols, generator=g, device=DEV).to(TYPES[kind])
        out = lambda: torch.empty(tokens, rows, device=DEV)
        want = lc.q4_matvec(q4, x, out())
        for bad in (float("inf"), float("nan"), big):
            for at in {0, tokens // 2, tokens - 1}:
                y = x.clone()
                y[at, ::7] = bad
                got = lc.q4_matvec(q4, y, out())
                others = [t for t in range(tokens) if t != at]
                assert torch.equal(got[others], want[others]), (tokens, bad, at)
                if bad != big:
                    assert not bool(got[at].isfinite().any())
                else:  # what the formula says, in 64 bits, where fp32 holds it
                    exact = y[at].double() @ lc.q4_read(q4).double().T
                    size = y[at].double().abs() @ lc.q4_read(q4).double().abs().T
                    holds = exact.abs() < 2.0 ** 127
                    near = (got[at].double() - exact).abs() <= size * (17 * group / 16 * 2.0 ** -23 + (cols / group + 16) * 2.0 ** -24)
                    assert kind != "fp16" or bool((near | ~holds).all())
