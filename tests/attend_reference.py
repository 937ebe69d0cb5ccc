"""Attention to a quantised cache, and the plan of a step, from the text of lc.h in 64 bits. Shares nothing with the CUDA library but
quant_reference's groups and codes."""
import numpy as np
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def attend(q, k, v, positions, scale, cap=0.0, slopes=None, window=0, prefix=0):
    """One sequence: q [n, heads, dim], k and v [length, cache heads, dim], all float64; positions [n]. Returns out, and what an error bound needs: the
    mean of |v| under the probabilities (like out), and for every row and head the largest sum of |q k| and |slope| * distance of its visible keys."""
    n, heads, dim = q.shape
    length, shared = k.shape[0], heads // k.shape[1]
    at = torch.arange(length, device=q.device)
    away = positions[:, None] - at[None, :]
    seen = (away >= 0) & ((away < window) if window else True) | (at[None, :] < prefix)
    out, size, plain = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    products, bias = torch.zeros(n, heads, dtype=torch.float64, device=q.device), torch.zeros(n, heads, dtype=torch.float64, device=q.device)
    for h in range(heads):
        kk, vv = k[:, h // shared], v[:, h // shared]
        t = scale * (q[:, h] @ kk.T)
        products[:, h] = (abs(scale) * (q[:, h].abs() @ kk.abs().T)).masked_fill(~seen, 0.0).amax(-1)
        if cap:
            t = cap * torch.tanh(t / cap)
        if slopes is not None:
            t = t - slopes[h].double() * away.abs()
            near = torch.where(t > t.masked_fill(~seen, -torch.inf).amax(-1, keepdim=True) - 20.0, away.abs().double(), 0.0)
            bias[:, h] = abs(float(slopes[h])) * near.masked_fill(~seen, 0.0).amax(-1)
        t = t.masked_fill(~seen, -torch.inf)
        p = torch.exp(t - t.amax(-1, keepdim=True))
        p = torch.where(seen, p, 0.0)
        total = p.sum(-1, keepdim=True)
        hidden = lambda x: torch.where(seen.any(0)[:, None], x, 0.0)
        out[:, h] = (p @ hidden(vv)) / total
        size[:, h] = (p @ hidden(vv.abs())) / total
        plain[:, h] = seen.double() @ hidden(vv.abs())
    return out, size, products, bias, plain


def bound(kind, out, size, products, bias, plain, dim, cap=0.0):
    """How far an output may be off, for a type whose products are rounded as lc.h says. With u half a step of the type (2^-8 for bf16): keys
    rounded to the type move a score by u * sum |q k|, sums in fp32 by (dim + 32) 2^-24 of that, a bias by 2^-22 of its size (keys that it lowers
    by 20 or more do not count: they weigh e^-20 together with their error); the cap halves none of this and its own function is good to cap * 2^-20; exp
    is good to 2^-20. A score that is off by d moves its weight by d of itself, and so does the sum that divides: 2 d. Probabilities and values
    rounded to the type: 2 u of the mean of |v|; the result's own rounding: u of itself. A small probability that is held in fp16 (of bf16 rows too) has fewer bits: 2^7 times as large beside a largest one of 1 or
    more, it is on a grid of 2^-24 at worst, so off by 2^-25 / 2^7 of the largest, and so of their sum: 2^-32 for every |v| that is seen. Values in fp16 are in units of a power of two near their block's largest scale
    and keep its 11 bits, no fewer than their rows' type, while no scale is 2^14 times as small; so they have no term of their own here."""
    u = HALF_STEP[kind]
    given = 0.0 if kind == torch.float32 else u
    d = (given + (dim + 32) * 2.0 ** -24) * products + 2.0 ** -22 * bias + cap * 2.0 ** -20 + 2.0 ** -20
    d = torch.expm1(d)[..., None]  # for scores that are off by much
    return (2 * max(given, 2.0 ** -22) + 2 * d) * size * 1.01 + u * out.abs() * 1.01 + 2.0 ** -24 * (kind == torch.float16) + 2.0 ** -32 * plain * (kind != torch.float32) + 1e-30


def plan(table, held, spare, count, tokens, page, rows):
    """(begin, first, slots, held, count, table, spare) after a step, or None if it does not fit; lists and numpy arrays of whole numbers."""
    table, spare = table.copy(), spare.copy()
    n, width = table.shape
    if count < 0 or count > len(spare) or any(h < 0 or h > width * page for h in held):
        return None
    if any(t > 0 and h + t > width * page for h, t in zip(held, tokens)):
        return None
    back = [table[s, j] for s in range(n) if tokens[s] < 0 for j in range(-(-held[s] // page))]
    if count + len(back) > len(spare):
        return None
    spare[count : count + len(back)] = back
    count += len(back)
    begin, first, slots, after = [0], [], [], []
    for s in range(n):
        first.append(0 if tokens[s] < 0 else int(held[s]))
        after.append(first[s] + max(0, int(tokens[s])))
        for j in range(-(-first[s] // page), -(-after[s] // page)):
            count -= 1
            if count < 0:
                return None
            table[s, j] = spare[count]
        slots += [int(table[s, p // page]) * page + p % page for p in range(first[s], after[s])]
        begin.append(len(slots))
    if len(slots) > rows:
        return None
    return begin, first, slots + [-1] * (rows - len(slots)), after, count, table, spare
