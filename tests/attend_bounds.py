"""How far attention to a quantised cache may be off, from what each of its roundings does, key by key; against what a mistake in the formula would do.

An output is sum p_k v_k with weights p_k of sum 1. A score that is off by d_k makes p_k of it p_k e^d_k, over a sum that changes likewise, and as sum p_k (v_k - out) is 0, the
output moves by no more than

    sum p_k |e^d_k - 1| |v_k - out| / sum p_k e^-|d_k|

A score is off by what its key's rounding and its sums in fp32 do. With u = 2^-11, half a step of 11 bits, beside 1:
* `many` (sequences of more than 16 rows for a head of the cache, in 16 bits, dim at most 128): keys of 8-bit codes have 11 bits: u sum |q k|. (Codes of 4 bits times a scale of 8 are exact in 11.)
  Queries of bf16 are held to 2^-25 of the largest of their row: 2^-25 max |q| sum |k|. In the other kernel neither is rounded.
* sums of dim products: (dim + 32) 2^-24 sum |q k|. exp, and its argument's rounding: 2^-20 + 2^-22 |t|. A bias: 2^-22 of itself. A cap: 2^-20 of the score, or 2^-16 with up to 64 in 16 bits.

Weights and values, relative to sum p |v|: weights have 11 bits where `many`, else what the rows' type has twice over (bf16 8 bits, fp16 16, fp32 24); values of 8-bit codes 11 where
`many`. Sums over n keys in fp32, 16 at a time: n 2^-27 of sum p |v|, and n 2^-25 of the output for the sum that divides. Small weights in fp16, 2^7 times as large as the largest is at least, are on a grid
of 2^-24: off by 2^-32 for every |v| that is seen. (`apart`: where scales differ by 2^14 and more, weights take the power of two that a key's values have beside the row's
largest weighted ones, so that 2^-32 is of those: with codes of at most c, and a scale's power of two in half a scale at least, off by 2^-31 of max_k p_k |v_k| for every key.)
A key that may move its own weight by e^20 makes a row's bound infinite. The result's own rounding comes last.

Where all those roundings are independent of each other the mean square is known too: a number rounded to half a step h of itself at most is off by h^2 / 3 in the mean at most. (A score in fp32
is summed 16 products at a time, those of fp32 queries in three parts, and each of these 3 dim / 16 sums is off by 2^-23 of sum |q k| at most. Of fp32 rows that is the most of it.)
"""
import torch


def telling(q, k, positions):
    """Queries like q (noise of size 1) that the keys on both sides of a mask's borders matter to: the sequence's first one, a row's own and the one behind it, each about as much
    as some thousand others (for scores of 2 / sqrt(dim) times the products). A mask that is off by one then shows."""
    unit = k / k.norm(dim=-1, keepdim=True).clamp(min=1e-30)
    shared = q.shape[1] // k.shape[1]
    behind = (positions + 1).clamp(max=k.shape[0] - 1)
    return q + 5.0 * (unit[positions] + unit[behind] + unit[:1]).repeat_interleave(shared, 1)


HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
U = 2.0 ** -11


def attend(kind, bits, many, q, k, v, positions, scale, cap=0.0, slopes=None, window=0, prefix=0, apart=False):
    """One sequence (as in attend_reference.attend): out, how far off it may be, and its mean square."""
    n, heads, dim = q.shape
    length, shared = k.shape[0], heads // k.shape[1]
    at = torch.arange(length, device=q.device)
    away = positions[:, None] - at[None, :]
    seen = (away >= 0) & ((away < window) if window else True) | (at[None, :] < prefix)
    some = seen.any(0)
    key = U if many and bits == 8 else 0.0
    steps = 3 * -(-dim // 16)
    weight = U if many else {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -16, torch.float32: 2.0 ** -24}[kind]
    out, allowed, square = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    for h in range(heads):
        qq, kk = q[:, h], torch.where(some[:, None], k[:, h // shared], 0.0)
        vv = torch.where(some[:, None], v[:, h // shared], 0.0)
        t = scale * (qq @ kk.T)
        products = abs(scale) * (qq.abs() @ kk.abs().T)
        d = (key + (dim + 32) * 2.0 ** -24) * products + 2.0 ** -20
        if many and kind == torch.bfloat16:
            d = d + 2.0 ** -25 * abs(scale) * qq.abs().amax(-1)[:, None] * kk.abs().sum(-1)[None, :]
        if cap:
            d = d + 2.0 ** -20 * t.abs() + (2.0 ** -16 if cap <= 64 and kind != torch.float32 else 0.0)
            t = cap * torch.tanh(t / cap)
        if slopes is not None:
            t = t - slopes[h].double() * away.abs()
            d = d + 2.0 ** -22 * slopes[h].double().abs() * away.abs()
        d = d + 2.0 ** -22 * t.abs()
        wild = (seen & (d > 20.0)).any(-1)
        d = d.clamp(max=20.0)
        t = t.masked_fill(~seen, -torch.inf)
        p = torch.where(seen, torch.exp(t - t.amax(-1, keepdim=True)), 0.0)
        p = p / p.sum(-1, keepdim=True)
        out[:, h] = o = p @ vv
        moved = p * torch.expm1(d)
        size = p @ vv.abs()
        off = (moved @ vv.abs() + o.abs() * moved.sum(-1, keepdim=True)) / (p * torch.exp(-d)).sum(-1, keepdim=True)
        off += (weight + key + length * 2.0 ** -27 + 2.0 ** -20) * size + length * 2.0 ** -25 * o.abs()
        if many:
            off += 2.0 ** -32 * seen.double() @ vv.abs()
        if many and apart:
            off += 2.0 ** -31 * (p * vv.abs().amax(-1)).amax(-1, keepdim=True) * seen.sum(-1, keepdim=True)
        off = off.masked_fill(wild[:, None], torch.inf)
        allowed[:, h] = 1.01 * (off + HALF_STEP[kind] * (o.abs() + off)) + (2.0 ** -24 if kind == torch.float16 else 1e-30)
        spread = p ** 2 * ((key * scale) ** 2 / 3 * (qq ** 2 @ (kk ** 2).T) + steps * (2.0 ** -23 * products) ** 2)
        square[:, h] = spread @ vv ** 2 - 2 * o * (spread @ vv) + o ** 2 * spread.sum(-1, keepdim=True)
        square[:, h] += (weight ** 2 + key ** 2) / 3 * (p ** 2 @ vv ** 2) + (HALF_STEP[kind] * o) ** 2 / 3 + (2.0 ** -20 * size) ** 2
    return out, allowed, square
