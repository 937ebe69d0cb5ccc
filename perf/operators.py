"""The operators on model state in few bits, as timed cases: their plain forms, and the calls that a program makes of them.

A program that recovers a model from its checkpoints serves it with weights in 4 bits and keeps a cache of keys and
values in 8 or 4. Both hold groups of consecutive values as whole numbers with a scale: with Q = 7 for 4 bits and 127 for
8, a group's scale is the largest magnitude over Q, rounded once to bfloat16, and a value's code the nearest whole number
of its quotient with that scale (ties to even). What a code stands for is its product with the scale.

* ``quantize``: a weight matrix into 4 bits, and back into numbers (a layer that is checked after it was quantised).
* ``matvec``: products of 4-bit weights with the vectors of one or a few tokens.
* ``write``: keys and values of new tokens into the slots of a cache, and the same rows read back.
* ``read``: sequences of different lengths out of a cache of pages, one behind the other.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
# the largest listed matrices and batch of sequences, in values: what is drawn stays below
LARGEST_PRODUCT, LARGEST_QUANTIZED, LARGEST_READ = 28672 * 8192, 4096 * 25088, 24 * 8192 * 8 * 128


def listed():
    return [
        # the first fully connected layer of the small convolutional state: one vector, nothing but latency
        {"name": "small layer", "op": "matvec", "rows": 120, "cols": 400, "tokens": 1, "type": "fp32", "group": 32, "pad": 0},
        # a square projection of a transformer, one token at a time
        {"name": "projection 1 token", "op": "matvec", "rows": 2048, "cols": 2048, "tokens": 1, "type": "bf16", "group": 128, "pad": 0},
        # the classifier behind a convolutional network's last feature map, a few images, in the state's own type
        {"name": "classifier 4 images", "op": "matvec", "rows": 4096, "cols": 25088, "tokens": 4, "type": "fp32", "group": 128, "pad": 0},
        # a batch of tokens through a layer of odd sizes, the vectors cut out of wider rows
        {"name": "odd layer 7 tokens", "op": "matvec", "rows": 8191, "cols": 5003, "tokens": 7, "type": "fp16", "group": 64, "pad": 6},
        # the scores over a vocabulary for a batch of sequences
        {"name": "vocabulary 16 tokens", "op": "matvec", "rows": 50257, "cols": 2048, "tokens": 16, "type": "bf16", "group": 64, "pad": 0},
        # a wide layer of a large model, one token: the weights are far larger than the L2 keeps
        {"name": "wide layer 1 token", "op": "matvec", "rows": 28672, "cols": 8192, "tokens": 1, "type": "bf16", "group": 128, "pad": 0},
        # one projection quantised after a recovery, and the largest layer of the convolutional state
        {"name": "quantize projection", "op": "quantize", "rows": 2048, "cols": 2048, "type": "fp32", "back": "bf16", "group": 64, "pad": 0},
        {"name": "quantize classifier", "op": "quantize", "rows": 4096, "cols": 25088, "type": "fp32", "back": "fp32", "group": 128, "pad": 0},
        # one step of a batch of sequences (some of them padding), and a long prompt
        {"name": "write a step", "op": "write", "tokens": 48, "heads": 8, "dim": 128, "bits": 8, "group": 128, "type": "bf16", "slots": 65536, "padding": 5},
        {"name": "write a prompt", "op": "write", "tokens": 16001, "heads": 8, "dim": 128, "bits": 4, "group": 32, "type": "fp16", "slots": 65536, "padding": 0},
        # a short prefix that is used again, and a batch of long sequences in pages
        {"name": "read a prefix", "op": "read", "sequences": 1, "longest": 200, "page": 16, "heads": 4, "dim": 80, "bits": 8, "group": 32, "type": "bf16"},
        {"name": "read a batch", "op": "read", "sequences": 24, "longest": 8192, "page": 64, "heads": 8, "dim": 128, "bits": 4, "group": 64, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    op = rng.choice(["matvec", "matvec", "matvec", "quantize", "write", "read"])
    case = {"op": op, "type": rng.choice(["bf16", "fp16", "fp32"]), "group": rng.choice([32, 64, 128])}
    if op in ("matvec", "quantize"):
        case["rows"] = _log(rng, 64, 32768)
        if op == "matvec":
            case["tokens"] = rng.choice([1, 1, 1, 2, 3, _log(rng, 1, 16), _log(rng, 1, 48)])
        most = min(LARGEST_PRODUCT, 4 * LARGEST_PRODUCT // case["tokens"]) if op == "matvec" else LARGEST_QUANTIZED
        case["cols"] = _log(rng, 48, min(32768, most // case["rows"]))
        if rng.random() < 0.6:  # most layers have even sizes
            case["rows"] -= case["rows"] % 16
            case["cols"] -= case["cols"] % 16
        case["pad"] = rng.choice([0, 0, 8, 3])
        if op == "quantize":
            case["back"] = rng.choice(["bf16", "fp16", "fp32"])
        return case
    case["heads"] = rng.choice([1, 2, 4, 8, 10])
    case["dim"] = rng.choice([64, 80, 96, 128, 128, 256, 100, 49])
    case["bits"] = rng.choice([4, 8])
    if op == "write":
        case["tokens"] = _log(rng, 1, 8000)
        case["slots"] = 32768
        case["padding"] = rng.choice([0, 0, 3])
    else:
        case["sequences"] = _log(rng, 1, 24)
        values = case["sequences"] * case["heads"] * case["dim"] * (2 if case["type"] == "fp32" else 1)
        case["longest"] = _log(rng, 8, min(8192, LARGEST_READ // values))
        case["page"] = rng.choice([1, 16, 64, 100])
    return case


def _random(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 100_003 + 17)
    return g


def _weights(case, g):
    """Rows of different spread, as a layer's; a strided view where the matrix is part of a wider one."""
    rows, cols, pad = case["rows"], case["cols"], case["pad"]
    spread = 0.02 * torch.exp(0.3 * torch.randn(rows, 1, generator=g, device=DEVICE))
    w = torch.randn(rows, cols + pad, generator=g, device=DEVICE) * spread
    return w[:, :cols]


def _tokens(case, g):
    """Activations: a few channels much larger than the others."""
    cols, pad = case["cols"], case["pad"]
    channel = 1.0 + 20.0 * (torch.rand(cols + pad, generator=g, device=DEVICE) < 0.002)
    x = torch.randn(case["tokens"], cols + pad, generator=g, device=DEVICE) * channel
    return x.to(TYPES[case["type"]])[:, :cols]


def _keys_values(case, n, g):
    """Keys and values of n tokens as a joint projection leaves them: side by side in the rows of one tensor."""
    heads, dim = case["heads"], case["dim"]
    joint = torch.randn(n, 2 * heads, dim, generator=g, device=DEVICE)
    joint[:, :heads] += 3.0 * torch.randn(heads, dim, generator=g, device=DEVICE)  # keys have channels off zero
    joint = joint.to(TYPES[case["type"]])
    return joint[:, :heads], joint[:, heads:]


def _slots(case, g):
    """Distinct slots for the tokens; -1 for those that only fill the batch up."""
    slots = torch.randperm(case["slots"], generator=g, device=DEVICE)[: case["tokens"]]
    pad = min(case["padding"], case["tokens"])
    slots[case["tokens"] - pad :] = -1
    return slots


def _pages(case, g):
    """A batch of sequences: (table of pages, first output row of each sequence and their end, rows, pages). The lengths go by
    the case, so that a pass has the same size with every seed; the seed deals out the pages."""
    n, longest, page = case["sequences"], case["longest"], case["page"]
    r = np.random.RandomState(n * 10_007 + longest)
    lengths = r.randint(max(1, longest // 3), longest + 1, n)
    lengths[0] = longest
    begin = np.concatenate([[0], np.cumsum(lengths)])
    width = -(-longest // page)
    order = torch.randperm(n * width + 3, generator=g, device=DEVICE)[: n * width]
    return order.to(torch.int32).view(n, width), torch.tensor(begin, dtype=torch.int32, device=DEVICE), int(begin[-1]), n * width + 3


def _groups(x, group):
    """x with its last axis cut into groups, the last one filled up with zeros."""
    n = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -n % group)).unflatten(-1, (-1, group))


def _quantized(x, bits, group):
    """(codes as int8, scales as float32), the definition by elementary operations. The quotients are taken in 64 bits: next to a
    border between two codes, or between two scales, 32 are not enough."""
    top = float(2 ** (bits - 1) - 1)
    g = _groups(x.float(), group)
    m, e = torch.frexp(g.abs().amax(-1).double() / top)
    s = torch.ldexp(torch.round(m * 256.0) / 256.0, e)
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    q = torch.where(s[..., None] > 0, torch.round(g.double() / s[..., None]), torch.zeros((), dtype=torch.float64, device=g.device))
    return q.to(torch.int8).flatten(-2)[..., : x.shape[-1]], s.float()


def _values(codes, scales, group):
    """What codes stand for, in float32 (exact)."""
    return (_groups(codes.float(), group) * scales[..., None]).flatten(-2)[..., : codes.shape[-1]]


def prepare(case, seed):
    op, group, g = case["op"], case["group"], _random(seed)
    t = TYPES[case["type"]]
    s = {"op": op, "case": case}
    if op == "matvec":
        w = _weights(case, g)
        s["x"] = _tokens(case, g)
        s["out"] = torch.empty(case["tokens"], case["rows"], dtype=t, device=DEVICE)
        if own:
            from paper_2009_13003_b200 import binding

            s["weights"] = binding.q4_quantize(w, group)
        else:
            s["codes"], s["scales"] = _quantized(w, 4, group)
        return s
    if op == "quantize":
        s["w"] = _weights(case, g).to(t)
        s["out"] = torch.empty(case["rows"], case["cols"], dtype=TYPES[case["back"]], device=DEVICE)
        if own:
            from paper_2009_13003_b200 import binding

            s["weights"] = binding.alloc_q4(case["rows"], case["cols"], group, DEVICE)
            s["workspace"] = binding.alloc_workspace(0, DEVICE)
        return s
    heads, dim, bits = case["heads"], case["dim"], case["bits"]
    if op == "write":
        s["k"], s["v"] = _keys_values(case, case["tokens"], g)
        s["slots"], rows, slots = _slots(case, g), case["tokens"], case["slots"]
    else:
        s["table"], s["begin"], rows, pages = _pages(case, g)
        slots = pages * case["page"]
        k, v = _keys_values(case, slots, g)
    # the rows of tokens that only fill the batch up stay as they are here
    s["out"] = [torch.zeros(rows, heads, dim, dtype=t, device=DEVICE) for _ in range(2)]
    if own:
        from paper_2009_13003_b200 import binding

        s["cache"] = binding.alloc_cache(slots, heads, dim, bits, group, DEVICE)
        if op == "read":
            binding.cache_write(s["cache"], k, v, torch.arange(slots, device=DEVICE))
    elif op == "write":  # one slot more than there are, which takes what belongs to none
        s["codes"] = torch.zeros(2, slots + 1, heads, dim, dtype=torch.int8, device=DEVICE)
        s["scales"] = torch.zeros(2, slots + 1, heads, -(-dim // group), device=DEVICE)
    else:
        s["codes"], s["scales"] = _quantized(torch.stack([k, v]), bits, group)
    return s


def _run_plain(s):
    op, case = s["op"], s["case"]
    group, t = case["group"], TYPES[case["type"]]
    if op == "matvec":
        return (s["x"].float() @ _values(s["codes"], s["scales"], group).T).to(t)
    if op == "quantize":
        return _values(*_quantized(s["w"], 4, group), group).to(TYPES[case["back"]])
    if op == "write":
        slots = s["slots"]
        codes, scales = _quantized(torch.stack([s["k"], s["v"]]), case["bits"], group)
        s["codes"][:, slots] = codes
        s["scales"][:, slots] = scales
        values = _values(s["codes"][:, slots], s["scales"][:, slots], group).to(t)
        k, v = torch.where((slots >= 0)[:, None, None], values, torch.stack(s["out"]))
        return k, v
    # the sequence of every row, its place in there, the page that holds it
    begin, page = s["begin"].long(), case["page"]
    row = torch.arange(s["out"][0].shape[0], device=DEVICE)
    seq = (row[:, None] >= begin[None, 1:]).sum(1)
    at = row - begin[seq]
    slots = s["table"][seq, at // page].long() * page + at % page
    k, v = _values(s["codes"][:, slots], s["scales"][:, slots], group).to(t)
    return k, v


def run(s):
    if not own:
        return _run_plain(s)
    from paper_2009_13003_b200 import binding

    op = s["op"]
    if op == "matvec":
        return binding.q4_matvec(s["weights"], s["x"], s["out"])
    if op == "quantize":
        binding.q4_quantize_async(s["w"], s["weights"], s["workspace"])
        return binding.q4_read(s["weights"], s["out"])
    if op == "write":
        binding.cache_write(s["cache"], s["k"], s["v"], s["slots"])
        return tuple(binding.cache_read(s["cache"], s["slots"], s["out"]))
    return tuple(binding.cache_read_pages(s["cache"], s["table"], s["case"]["page"], s["begin"], s["out"]))


def _held(n, bits, group):
    """Bytes that a row of n values takes: codes and scales."""
    return n * bits / 8 + 2 * math.ceil(n / group)


def work(case):
    op, size = case["op"], SIZE[case["type"]]
    if op == "matvec":
        rows, cols, tokens = case["rows"], case["cols"], case["tokens"]
        return {"bytes": rows * _held(cols, 4, case["group"]) + tokens * (rows + cols) * size, "flops": 2 * tokens * rows * cols}
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size + SIZE[case["back"]]) + 2 * case["rows"] * _held(case["cols"], 4, case["group"]), "flops": 4 * n}
    heads, dim = case["heads"], case["dim"]
    rows = case["tokens"] if op == "write" else case["sequences"] * case["longest"] * 2 / 3
    held = 2 * rows * heads * _held(dim, case["bits"], case["group"])
    plain = 2 * rows * heads * dim * size
    return {"bytes": 2 * (held + plain) + 16 * rows if op == "write" else held + plain + 4 * rows / case["page"], "flops": 2 * rows * heads * dim}


def _nearest(x, bits, group):
    """The definition in 64 bits: every value's nearest multiple of its group's scale."""
    x = x.double()
    top, n = 2 ** (bits - 1) - 1, x.shape[-1]
    out = torch.empty_like(x)
    for lo in range(0, n, group):
        part = x[..., lo : lo + group]
        most = part.abs().max(dim=-1, keepdim=True).values / top
        unit = torch.exp2(torch.floor(torch.log2(most.clamp(min=1e-300))) - 7)  # what the last of 8 significant bits counts for
        unit = torch.where(most / unit >= 256, 2 * unit, torch.where(most / unit < 128, unit / 2, unit))
        low = torch.floor(most / unit)
        rest = most / unit - low
        scale = (low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 == 1)))) * unit
        scale = torch.where(scale < 2.0 ** -126, 0.0 * scale, scale)
        y = part / torch.where(scale > 0, scale, torch.ones_like(scale))
        low = torch.floor(y)
        rest = y - low
        out[..., lo : lo + group] = (low + ((rest > 0.5) | ((rest == 0.5) & (low.remainder(2) == 1)))) * scale
    return out


def exact(case, seed):
    op, group, g = case["op"], case["group"], _random(seed)
    if op == "matvec":
        w = _nearest(_weights(case, g), 4, group)
        return _tokens(case, g).double() @ w.T
    if op == "quantize":
        return _nearest(_weights(case, g).to(TYPES[case["type"]]), 4, group)
    if op == "write":
        k, v = _keys_values(case, case["tokens"], g)
        none = (_slots(case, g) < 0)[:, None, None]
        return tuple(_nearest(x, case["bits"], group).masked_fill(none, 0.0) for x in (k, v))
    table, begin, rows, pages = _pages(case, g)
    k, v = _keys_values(case, pages * case["page"], g)
    first, page = begin.tolist(), case["page"]
    place = []
    for b in range(case["sequences"]):
        at = torch.arange(first[b + 1] - first[b], device=DEVICE)
        place.append(table[b].long()[at // page] * page + at % page)
    place = torch.cat(place)
    return tuple(_nearest(x[place], case["bits"], group) for x in (k, v))
