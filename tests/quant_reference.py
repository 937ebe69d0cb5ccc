"""docs/QUANT.md in 64 bits, from the text: groups, scales, codes, and the two layouts. NumPy on the CPU; shares nothing with the
CUDA library."""
import numpy as np


def bf16_bits(x):
    """Bit patterns of finite non-negative float64 values rounded once to bf16 (8 significant bits, subnormals on their grid)."""
    x = np.asarray(x, np.float64)
    m, e = np.frexp(x)
    unit = np.ldexp(1.0, np.maximum(e - 8, -133))  # what the last bit counts for
    r = np.rint(x / unit) * unit  # rint: ties to even; the division by a power of two is exact
    return (r.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def bf16_values(bits):
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def groups(x, group):
    n = x.shape[-1]
    pad = -n % group
    return np.pad(x, [(0, 0)] * (x.ndim - 1) + [(0, pad)]).reshape(x.shape[:-1] + ((n + pad) // group, group))


def quantize(x, bits, group):
    """(codes, scale bits) of float32 (or narrower) values given as float64."""
    top = 2 ** (bits - 1) - 1
    g = groups(np.asarray(x, np.float64), group)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    # the quotients of numbers of 24 bits are at least 2^-33 (relative) away from a border or on it: 64 bits decide it
    s = bf16_bits(np.abs(g).max(-1) / top)
    s = np.where(s < 0x0080, 0, s).astype(np.uint16)
    v = bf16_values(s)[..., None]
    q = np.where(v > 0, np.rint(g / np.where(v > 0, v, 1.0)), 0.0).astype(np.int64)
    s = np.where(bad, 0x7FC0, s).astype(np.uint16)
    n = x.shape[-1]
    return q.reshape(q.shape[:-2] + (-1,))[..., :n], s


def values(codes, scale_bits, group):
    n = codes.shape[-1]
    v = groups(codes.astype(np.float64), group) * bf16_values(scale_bits)[..., None]
    return v.reshape(v.shape[:-2] + (-1,))[..., :n]


def q4_bytes(rows, cols, group):
    t, s = -(-rows // 16), -(-cols // 128)
    return -(-(1024 * t * s + 32 * t * (128 * s // group)) // 256) * 256


def q4_unpack(data, rows, cols, group):
    """(codes, scale bits) of the whole tiles and steps in a buffer of 4-bit weights (section 2)."""
    t, s = -(-rows // 16), -(-cols // 128)
    words = data[: 1024 * t * s].view(np.uint32).reshape(t, 2 * s, 8, 4, 2, 2)  # tile, block, r, t, h, j
    codes = np.zeros((t, 16, 2 * s, 2, 4, 2, 4), np.int64)  # tile, row, block, h, t, j, column
    for p in range(4):
        for e in range(2):
            v = ((words >> np.uint32(4 * p + 16 * e)) & np.uint32(15)).astype(np.int64) - 8
            codes[:, 8 * (p % 2) : 8 * (p % 2) + 8, :, :, :, :, 2 * (p // 2) + e] = v.transpose(0, 2, 1, 4, 3, 5)
    n = 128 * s // group
    scales = data[1024 * t * s : 1024 * t * s + 32 * t * n].view(np.uint16).reshape(t, n, 8, 2).transpose(0, 3, 2, 1)
    return codes.reshape(16 * t, 128 * s), scales.reshape(16 * t, n)


def cache_unpack(codes, dim, bits):
    """Codes of the rows of a cache (section 3), from bytes [..., row]."""
    if bits == 8:
        return codes[..., :dim].astype(np.int64) - 128
    w = np.ascontiguousarray(codes).view("<u4")
    e = np.arange(8, dtype=np.uint32)
    v = (w[..., None] >> (4 * (e // 2) + 16 * (e % 2)).astype(np.uint32)) & np.uint32(15)
    return v.reshape(v.shape[:-2] + (-1,))[..., :dim].astype(np.int64) - 8
