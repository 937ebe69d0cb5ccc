"""Attention over a quantised cache in pages, and the plan of a step, as timed cases: their plain forms, and the calls that a program makes of them.

A program that serves a recovered model keeps the keys and values of its sequences in a cache of pages. Every step brings new tokens
for some of the sequences: they get pages and slots, their keys and values go there, and they attend to what the cache holds.

* ``plan``: from the numbers of new tokens of all sequences, where each one's rows begin in the batch, the pages that it needs beyond those it
  has (taken off a list of spare ones, to which those of sequences that end go back), and the slot of every new token.
* ``attend``: the new tokens' attention to the cache. A query at position i of its sequence sees the positions p <= i (with a window, only
  the last ones), and with a prefix also all of that. Scores may be capped (cap * tanh(score / cap)) and lowered by slope * |i - p|. Several
  heads of the queries share one of the cache.

A cache holds groups of consecutive values as whole numbers with a scale: with Q = 7 for 4 bits and 127 for 8, a group's scale is the
largest magnitude over Q, rounded once to bfloat16, and a value's code the nearest whole number of its quotient with that scale (ties to
even). What a code stands for is its product with the scale.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}

_ATTEND = {"op": "attend", "page": 16, "cap": 0.0, "slopes": False, "window": 0, "prefix": 0, "chunks": 0, "drafts": 1}


def listed():
    return [
        # one step of a batch of sequences, a token each; some wait, some have ended
        {"name": "plan a step", "op": "plan", "sequences": 48, "longest": 4096, "prompts": 0, "prompt": 0, "page": 16, "spare_rows": 0},
        # a step with some prompts among the single tokens, in a batch of fixed size that it does not fill
        {"name": "plan a mixed step", "op": "plan", "sequences": 256, "longest": 8192, "prompts": 9, "prompt": 3001, "page": 64, "spare_rows": 777},
        # many sequences begin at once, in small pages
        {"name": "plan prompts", "op": "plan", "sequences": 2048, "longest": 300, "prompts": 2048, "prompt": 512, "page": 16, "spare_rows": 0},
        # the first token behind a short prompt: nothing but latency
        dict(_ATTEND, name="a token, short", sequences=1, longest=200, heads=4, shared=1, dim=80, bits=8, group=32, type="bf16"),
        # a token for each sequence of a batch, over the cache in 4 bits
        dict(_ATTEND, name="a token, batch", sequences=24, longest=8192, page=64, heads=8, shared=4, dim=128, bits=4, group=64, type="bf16"),
        # a token for each of a few very long sequences
        dict(_ATTEND, name="a token, long", sequences=3, longest=131072, page=64, heads=8, shared=8, dim=128, bits=8, group=128, type="bf16"),
        # drafted tokens that are checked together, wide heads, capped scores
        dict(_ATTEND, name="drafts, capped", sequences=16, longest=3001, heads=4, shared=2, dim=256, bits=8, group=128, type="fp16", drafts=5, cap=50.0),
        # a long prompt taken in parts: the next part of two of them
        dict(_ATTEND, name="chunks", sequences=2, longest=16384, page=64, heads=8, shared=4, dim=128, bits=8, group=128, type="bf16", chunks=2, drafts=1024),
        # a whole prompt at once
        dict(_ATTEND, name="a prompt", sequences=1, longest=8192, page=64, heads=8, shared=4, dim=128, bits=8, group=128, type="bf16", chunks=1, drafts=8192),
        # single tokens and parts of prompts in one step
        dict(_ATTEND, name="mixed step", sequences=32, longest=6000, page=16, heads=8, shared=4, dim=128, bits=4, group=32, type="fp16", chunks=2, drafts=1000),
        # short prompts of a model that lowers scores by distance, every head with its own keys
        dict(_ATTEND, name="prompts, slopes", sequences=5, longest=2500, heads=12, shared=1, dim=64, bits=8, group=64, type="bf16", chunks=5, drafts=2500, slopes=True),
        # a picture that is seen as a whole ahead of text in a window
        dict(_ATTEND, name="picture and text", sequences=3, longest=3700, page=100, heads=6, shared=2, dim=96, bits=8, group=32, type="fp16", chunks=3, drafts=3700,
             window=512, prefix=1024),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    if rng.random() < 0.25:
        n = _log(rng, 1, 2048)
        longest = _log(rng, 16, min(8192, 1200000 // n))
        prompts = rng.choice([0, 0, _log(rng, 1, n), n])
        return {"op": "plan", "sequences": n, "longest": longest, "prompts": prompts, "prompt": _log(rng, 2, min(4096, max(2, 1000000 // n))),
                "page": rng.choice([1, 16, 16, 32, 64, 100]), "spare_rows": rng.choice([0, 5, 1000])}
    case = dict(_ATTEND)
    case["type"] = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
    case["bits"], case["group"] = rng.choice([4, 8]), rng.choice([32, 64, 128])
    case["heads"], case["shared"] = rng.choice([(1, 8), (2, 4), (4, 1), (8, 4), (8, 8), (12, 1), (4, 7), (6, 2)])
    case["dim"] = rng.choice([64, 80, 96, 128, 128, 128, 256, 100, 49])
    case["page"] = rng.choice([1, 16, 16, 64, 64, 100])
    case["cap"] = rng.choice([0.0, 0.0, 0.0, 30.0])
    case["slopes"] = rng.random() < 0.2
    case["window"] = rng.choice([0, 0, 0, 128, 1000])
    case["prefix"] = rng.choice([0, 0, 0, 4, 500])
    kind = rng.choice(["tokens", "tokens", "drafts", "chunks", "prompts", "mixed"])
    if case["type"] == "fp32" and kind in ("chunks", "prompts", "mixed"):
        kind = "drafts"  # prompts come in 16 bits
    width = case["heads"] * case["dim"]
    if kind in ("tokens", "drafts"):
        case["sequences"] = _log(rng, 1, 64)
        case["longest"] = _log(rng, 16, min(100000, 250000000 // (case["sequences"] * width)))
        case["drafts"] = 1 if kind == "tokens" else rng.randint(2, 9)
    else:
        # scores of all heads: no more than half of a prompt of 8192 with 32 heads
        most = 16 * 8192 * 8192 * 128 / (width * case["shared"])
        case["sequences"] = _log(rng, 1, 8) if kind != "mixed" else _log(rng, 2, 40)
        case["chunks"] = case["sequences"] if kind != "mixed" else rng.randint(1, min(3, case["sequences"]))
        case["longest"] = _log(rng, 64, min(16384, int(math.sqrt(most / case["chunks"]))))
        case["drafts"] = case["longest"] if kind == "prompts" else min(case["longest"], _log(rng, 17, 2048))
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------


def _random(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 100_003 + 29)
    return g


def _device(x):
    return torch.tensor(np.asarray(x, np.int32), dtype=torch.int32, device=DEVICE)


def _requests(case):
    """(held, new tokens) of every sequence of a plan: by the case, so that a pass has the same size with every seed."""
    n = case["sequences"]
    r = np.random.RandomState(n * 10_007 + case["longest"] + case["prompts"])
    held = r.randint(0, case["longest"] + 1, n)
    tokens = np.ones(n, np.int64)
    kind = r.rand(n)
    tokens[kind < 0.1] = 0  # waits
    tokens[kind > 0.93] = -1  # has ended
    begins = r.permutation(n)[: case["prompts"]]
    held[begins] = 0
    tokens[begins] = r.randint(max(1, case["prompt"] // 3), case["prompt"] + 1, len(begins))
    return held, tokens


def _books(case, seed):
    """The books of a plan: (held, tokens, table, spare pages, their number, rows of the batch), on the host."""
    held, tokens = _requests(case)
    page, n = case["page"], case["sequences"]
    width = -(-(case["longest"] + max(1, case["prompt"])) // page)
    has = -(-held // page)
    wants = -(-(held + np.maximum(tokens, 0)) // page)
    pages = int(has.sum() + (wants - has).sum() + 5)
    order = np.random.RandomState(seed % (1 << 31)).permutation(pages).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    taken = 0
    for s in range(n):
        table[s, : has[s]] = order[taken : taken + has[s]]
        taken += has[s]
    spare = np.full(pages, -1, np.int32)
    spare[: pages - taken] = order[taken:]
    return held, tokens, table, spare, pages - taken, int(np.maximum(tokens, 0).sum()) + case["spare_rows"]


def _batch(case):
    """(positions held ahead of the step, new tokens) of every sequence that attends, by the case."""
    n, longest = case["sequences"], case["longest"]
    r = np.random.RandomState(n * 10_007 + longest + case["drafts"])
    total = r.randint(max(1, longest // 3), longest + 1, n)
    total[0] = longest
    new = np.ones(n, np.int64) if case["chunks"] else np.full(n, case["drafts"])
    for s in range(case["chunks"]):  # the chunks stand at the end of the batch
        new[n - 1 - s] = max(1, case["drafts"] - 97 * s)
    if case["chunks"] == n and case["drafts"] >= longest:
        new = total.copy()  # whole prompts
    new = np.minimum(new, total)
    return total - new, new


def _keys_values(case, slots, g):
    """Keys and values of all slots, as a joint projection leaves them: side by side in the rows of one tensor."""
    heads, dim = case["heads"], case["dim"]
    joint = torch.randn(slots, 2 * heads, dim, generator=g, device=DEVICE)
    joint[:, :heads] += 2.0 * torch.randn(heads, dim, generator=g, device=DEVICE)  # keys have channels off zero
    joint = joint.to(TYPES[case["type"]])
    return joint[:, :heads], joint[:, heads:]


def _attending(case, seed):
    """What a step attends with: (host lengths, tables, keys, values, queries, slopes)."""
    g = _random(seed)
    first, new = _batch(case)
    n, page, heads, dim = case["sequences"], case["page"], case["heads"], case["dim"]
    width = -(-case["longest"] // page)
    used = -(-(first + new) // page)
    pages = int(used.sum()) + 3
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for s in range(n):
        table[s, : used[s]] = order[at : at + used[s]]
        at += int(used[s])
    k, v = _keys_values(case, pages * page, g)
    rows = int(new.sum())
    # queries as a projection leaves them beside something else
    q = torch.randn(rows, heads * case["shared"] + 2, dim, generator=g, device=DEVICE).to(TYPES[case["type"]])[:, : heads * case["shared"]]
    slopes = None
    if case["slopes"]:
        h = heads * case["shared"]
        slopes = torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device=DEVICE)
    return first, new, table, k, v, q, slopes


def _groups(x, group):
    """x with its last axis cut into groups, the last one filled up with zeros."""
    n = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -n % group)).unflatten(-1, (-1, group))


def _quantized(x, bits, group):
    """(codes as int8, scales as float32), the definition by elementary operations, quotients in 64 bits."""
    top = float(2 ** (bits - 1) - 1)
    g = _groups(x.float(), group)
    m, e = torch.frexp(g.abs().amax(-1).double() / top)
    s = torch.ldexp(torch.round(m * 256.0) / 256.0, e)
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    q = torch.where(s[..., None] > 0, torch.round(g.double() / s[..., None]), torch.zeros((), dtype=torch.float64, device=g.device))
    return q.to(torch.int8).flatten(-2)[..., : x.shape[-1]], s.float()


def _in_parts(x, bits, group):
    """_quantized, some rows at a time: the cache of a few long sequences is large."""
    parts = [_quantized(p, bits, group) for p in x.split(65536)]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def prepare(case, seed):
    s = {"op": case["op"], "case": case}
    if case["op"] == "plan":
        held, tokens, table, spare, count, rows = _books(case, seed)
        s["held"], s["tokens"], s["table"], s["spare"], s["count"], s["rows"] = _device(held), _device(tokens), _device(table), _device(spare), _device([count]), rows
        if own:
            from paper_2009_13003_b200 import binding

            s["pages"] = binding.Pages(s["table"], s["held"], s["spare"], s["count"], case["page"])
            # the books after the step go elsewhere, so that the same step can be planned again
            s["plan"] = binding.alloc_plan(s["pages"], rows, in_place=False)
            s["status"] = binding.alloc_status(DEVICE)
        return s
    first, new, s["table"], k, v, s["q"], s["slopes"] = _attending(case, seed)
    s["first"], s["begin"] = _device(first), _device(np.concatenate([[0], np.cumsum(new)]))
    s["prefix"] = _device(np.minimum(case["prefix"], first + new)) if case["prefix"] else None
    s["scale"] = 1.0 / math.sqrt(case["dim"])
    s["longest"] = int(new.max())
    s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
    if own:
        from paper_2009_13003_b200 import binding

        cache = s["cache"] = binding.alloc_cache(k.shape[0], case["heads"], case["dim"], case["bits"], case["group"], DEVICE)
        binding.cache_write(cache, k, v, torch.arange(k.shape[0], device=DEVICE))
        s["workspace"] = binding.alloc_attend_workspace(cache, case["sequences"])
        s["status"] = binding.alloc_status(DEVICE)
    else:
        s["new"], s["host"] = new.tolist(), first.tolist()  # a plain program knows its lengths
        s["k"], s["v"] = _in_parts(k, case["bits"], case["group"]), _in_parts(v, case["bits"], case["group"])
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------


def _plan_plain(s):
    page, table, held, spare = s["case"]["page"], s["table"].clone(), s["held"].long(), s["spare"].clone()
    n, width = table.shape
    tokens = s["tokens"].long()
    ends, new = tokens < 0, tokens.clamp(min=0)
    begin = torch.zeros(n + 1, dtype=torch.long, device=DEVICE)
    begin[1:] = new.cumsum(0)
    first = torch.where(ends, 0, held)
    after = first + new
    # pages of those that end go behind the spare ones
    column = torch.arange(width, device=DEVICE)
    count = s["count"].long()
    back = (ends[:, None] & (column < ((held + page - 1) // page)[:, None])).flatten().nonzero().squeeze(1)
    spare[count + torch.arange(back.numel(), device=DEVICE)] = table.flatten()[back]
    total = count + back.numel()
    # pages that are wanted come off the top
    wanted = (column >= ((first + page - 1) // page)[:, None]) & (column < ((after + page - 1) // page)[:, None])
    wanted = wanted.flatten().nonzero().squeeze(1)
    table.view(-1)[wanted] = spare[total - 1 - torch.arange(wanted.numel(), device=DEVICE)]
    row = torch.arange(s["rows"], device=DEVICE)
    seq = torch.searchsorted(begin[1:], row, right=True)
    real = seq < n
    seq = seq.clamp(max=n - 1)
    at = torch.where(real, first[seq] + row - begin[seq], 0)
    slots = torch.where(real, table[seq, at // page].long() * page + at % page, -1)
    return {"begin": begin.int(), "first": first.int(), "slots": slots, "held": after.int(), "count": (total - wanted.numel()).int(), "table": table, "spare": spare}


def _attend_plain(s):
    case, q, out = s["case"], s["q"], s["out"]
    page, group, shared, dim = case["page"], case["group"], case["shared"], case["dim"]
    row = 0
    for i, (held, n) in enumerate(zip(s["host"], s["new"])):
        length = held + n
        at = torch.arange(length, device=DEVICE)
        slots = s["table"][i, at // page].long() * page + at % page
        i_pos = held + torch.arange(n, device=DEVICE)
        away = i_pos[:, None] - at[None, :]
        seen = away >= 0
        if case["window"]:
            seen &= away < case["window"]
        if s["prefix"] is not None:
            seen |= at[None, :] < s["prefix"][i]
        for h in range(case["heads"]):
            k, v = (((_groups(c[slots, h].float(), group)) * sc[slots, h][..., None]).flatten(-2)[:, :dim] for c, sc in (s["k"], s["v"]))
            t = q[row : row + n, h * shared : (h + 1) * shared].float().transpose(0, 1) @ k.T * s["scale"]  # [shared, n, length]
            if case["cap"]:
                t = case["cap"] * torch.tanh(t / case["cap"])
            if s["slopes"] is not None:
                t -= s["slopes"][h * shared : (h + 1) * shared, None, None] * away.abs()
            t.masked_fill_(~seen, -math.inf)
            p = torch.exp(t - t.amax(-1, keepdim=True))
            out[row : row + n, h * shared : (h + 1) * shared] = ((p @ v) / p.sum(-1, keepdim=True)).transpose(0, 1).to(q.dtype)
        row += n
    return out


def run(s):
    if not own:
        return _plan_plain(s) if s["op"] == "plan" else _attend_plain(s)
    from paper_2009_13003_b200 import binding

    if s["op"] == "plan":
        plan = binding.cache_plan(s["pages"], s["tokens"], plan=s["plan"], status=s["status"])
        return {"begin": plan.begin, "first": plan.first, "slots": plan.slots, "held": plan.held, "count": plan.count, "table": s["table"], "spare": s["spare"]}
    case = s["case"]
    return binding.cache_attend(s["cache"], s["q"], s["table"], case["page"], s["begin"], s["out"], first=s["first"], scale=s["scale"], cap=case["cap"],
                                slopes=s["slopes"], window=case["window"], prefix=s["prefix"], longest=s["longest"], workspace=s["workspace"],
                                status=s["status"])


# ---- what a pass cannot do without, and the definition in 64 bits -------------------------------------------------


def _held(n, bits, group):
    """Bytes that a row of n values takes: codes and scales."""
    return n * bits / 8 + 2 * math.ceil(n / group)


def work(case):
    if case["op"] == "plan":
        held, tokens = _requests(case)
        page, new = case["page"], np.maximum(tokens, 0)
        pages = (-(-(held + new) // page) + held // -page).clip(0).sum() + (-(-held // page))[tokens < 0].sum()
        return {"bytes": float(20 * len(held) + 8 * (new.sum() + case["spare_rows"]) + 8 * pages), "flops": float(new.sum() + len(held))}
    first, new = _batch(case)
    window, heads, dim = case["window"] or 1 << 40, case["heads"], case["dim"]
    keys = pairs = 0
    for a, n in zip(first.tolist(), new.tolist()):
        prefix = min(case["prefix"], a + n)
        i = np.arange(a, a + n)
        low = np.maximum(i - window + 1, 0)
        # what lies at or ahead of a query in its window, and what of the prefix lies behind the query or ahead of the window
        pairs += int((i + 1 - low + np.maximum(prefix - i - 1, 0) + np.minimum(low, prefix)).sum())
        keys += a + n - max(int(low[0]) - prefix, 0)
    rows = int(new.sum()) * heads * case["shared"]
    return {"bytes": 2 * keys * heads * _held(dim, case["bits"], case["group"]) + 2 * rows * dim * SIZE[case["type"]],
            "flops": 4.0 * pairs * heads * case["shared"] * dim}


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


def _plan_exact(case, seed):
    held, tokens, table, spare, count, rows = _books(case, seed)
    page, n = case["page"], len(held)
    begin, first, slots = [0], [], []
    for s in range(n):
        if tokens[s] < 0:
            for j in range(-(-held[s] // page)):
                spare[count] = table[s, j]
                count += 1
    for s in range(n):
        first.append(0 if tokens[s] < 0 else int(held[s]))
        for p in range(first[s], first[s] + max(0, int(tokens[s]))):
            if p % page == 0:  # the first position of a page
                count -= 1
                table[s, p // page] = spare[count]
            slots.append(int(table[s, p // page]) * page + p % page)
        begin.append(len(slots))
    slots += [-1] * (rows - len(slots))
    after = [f + b - a for f, a, b in zip(first, begin, begin[1:])]
    return {"begin": _device(begin), "first": _device(first), "slots": torch.tensor(slots, dtype=torch.int64, device=DEVICE), "held": _device(after),
            "count": _device([count]), "table": _device(table), "spare": _device(spare)}


def exact(case, seed):
    if case["op"] == "plan":
        return _plan_exact(case, seed)
    first, new, table, k, v, q, slopes = _attending(case, seed)
    page, shared, window, cap = case["page"], case["shared"], case["window"], case["cap"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    row = 0
    for s in range(case["sequences"]):
        length, n = int(first[s] + new[s]), int(new[s])
        at = torch.arange(length, device=DEVICE)
        place = table[s].long().repeat_interleave(page)[:length] * page + at % page
        prefix = min(case["prefix"], length)
        for h in range(case["heads"]):
            keys, values = _nearest(k[place, h], case["bits"], case["group"]), _nearest(v[place, h], case["bits"], case["group"])
            for j in range(h * shared, (h + 1) * shared):
                for lo in range(0, n, 2048):
                    m = min(2048, n - lo)
                    i = (int(first[s]) + lo + torch.arange(m, device=DEVICE))[:, None]
                    t = (q[row + lo : row + lo + m, j].double() @ keys.T) / math.sqrt(case["dim"])
                    if cap:
                        t = torch.tanh(t / cap) * cap
                    if slopes is not None:
                        t = t - (i - at).abs() * slopes[j].double()
                    hidden = (at > i) | (at <= i - window) if window else at > i
                    t = torch.where(hidden & (at >= prefix), -math.inf, t)
                    out[row + lo : row + lo + m, j] = torch.softmax(t, -1) @ values
        row += n
    return out
