"""The bounds of attend_bounds hold for what the roundings that they name do, and for no mistake in the formula, nor for coarser roundings: on the CPU."""
import pytest
import torch

import attend_bounds as bounds
import attend_reference as ref

KINDS = [torch.bfloat16, torch.float16, torch.float32]


def numbers(kind, n, heads, shared, dim, length, seed):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(*shape, generator=g, dtype=torch.float64)
    k, v = (draw(length, heads, dim) * torch.exp(0.3 * draw(length, heads, 1)) for _ in range(2))
    at = length - n + torch.arange(n)
    return bounds.telling(draw(n, heads * shared, dim), k, at).to(kind).double(), k, v, at, 2.0 / dim ** 0.5


MISTAKES = ["zeros", "a key too few", "a key too many", "the first key is not seen", "a scale 1 % off", "keys one further", "heads the other way"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("many,n", [(False, 1), (False, 3), (True, 40)])
def test_mistakes_are_beyond(kind, many, n, dim):
    """A batch of sequences, as a test has it: each mistake is beyond the bound of some output or beyond the mean square of all."""
    many = many and kind != torch.float32
    far, squares, total = dict.fromkeys(MISTAKES, 0.0), dict.fromkeys(MISTAKES, 0.0), 0.0
    for length in (90, 300, 900, 1500, 2000, 3000):
        q, k, v, at, scale = numbers(kind, n, 1, 4, dim, length, length + n)
        out, allowed, square = bounds.attend(kind, 8, many, q, k, v, at, scale)
        own = ref.attend(q, k, v, at, scale)[0]
        assert torch.allclose(out, own, rtol=1e-12, atol=1e-12)
        rounded = own.to(kind).double()
        assert bool(((rounded - out).abs() <= allowed).all()) and float(((rounded - out) ** 2).sum()) <= float(square.sum())
        wrong = [torch.zeros_like(own), ref.attend(q, k, v, at - 1, scale)[0], ref.attend(q, k, v, at + 1, scale)[0], ref.attend(q, k, v, at, scale, window=length - n)[0],
                 ref.attend(q, k, v, at, 1.01 * scale)[0], ref.attend(q, torch.roll(k, 1, 0), v, at, scale)[0], own.flip(1)]
        total += float(square.sum())
        for name, got in zip(MISTAKES, wrong):
            far[name] = max(far[name], float(((got - out).abs() / allowed).max()))
            squares[name] += float(((got - out) ** 2).sum())
    for name in MISTAKES:
        if not (n == 1 and name == "a key too many"):  # a last row sees all keys
            assert far[name] > 1.5 or squares[name] > 1.5 * total, (name, far[name], squares[name] / total)


@pytest.mark.parametrize("kind", KINDS[:2])
@pytest.mark.parametrize("dim", [64, 128])
def test_coarser_roundings_are_beyond(kind, dim):
    """Keys, weights and values of 11 bits stay within; of 8 they are beyond the mean square."""
    q, k, v, at, scale = numbers(kind, 40, 1, 4, dim, 700, dim)
    out, allowed, square = bounds.attend(kind, 8, True, q, k, v, at, scale)

    def by(t):
        seen = at[:, None] >= torch.arange(700)[None, :]
        got = torch.zeros_like(out)
        for h in range(4):
            s = (scale * (q[:, h] @ k[:, 0].to(t).double().T)).masked_fill(~seen, -torch.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            got[:, h] = (p.to(t).double() @ v[:, 0].to(t).double()) / p.sum(-1, keepdim=True)
        return (got.to(kind).double() - out).abs()

    fine, coarse = by(torch.float16), by(torch.bfloat16)
    assert bool((fine <= allowed).all()) and float((fine ** 2).sum()) <= float(square.sum())
    assert float((coarse ** 2).sum()) > 1.3 * float(square.sum())
