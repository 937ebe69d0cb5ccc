"""How lc_q4_matvec lays products out: whatever the shape, there is a layout, and the kernel's areas of shared memory, worked out here as
the kernel does, stay within what the layout asks for (and that within an SM). CPU only."""
import ctypes as C
import itertools
import random

from paper_2009_13003_b200 import binding

NAMES = "per_pass nt mt ways split warps stages slice chunk direct smem".split()
MOST = 227 * 1024


def plan(rows, cols, group, kind, tokens, sms=148):
    out = (C.c_uint32 * len(NAMES))()
    assert binding.lib().lc_debug_q4_plan(rows, cols, group, kind, tokens, sms, out) == binding.OK
    return dict(zip(NAMES, out))


def check(rows, cols, group, kind, tokens, sms=148):
    p = plan(rows, cols, group, kind, tokens, sms)
    case = (rows, cols, group, kind, tokens, p)
    parts, steps = 3 if kind == 0 else 1, -(-cols // 128)
    columns = p["per_pass"] * parts
    assert 0 < p["smem"] <= MOST, case
    assert columns <= 8 * p["nt"] <= 32 and p["mt"] in (1, 2) and p["mt"] * p["nt"] <= 8, case
    assert p["ways"] in (1, 2, 4, 8) and p["split"] in (1, 2, 4, 8) and p["warps"] in (8, 16), case
    groups = p["warps"] // p["ways"]
    assert p["ways"] == 1 or groups <= 15, case  # a named barrier for each
    assert p["slice"] * p["split"] >= steps and p["slice"] >= 1 and 1 <= p["chunk"] <= p["slice"], case
    assert p["chunk"] == p["slice"] or p["chunk"] % p["ways"] == 0, case  # the order in which a ring is filled
    assert not p["direct"] or (p["ways"] == 1 and p["split"] == 1 and parts == 1), case
    assert 3 <= p["stages"] <= 6, case  # what the waits are made for
    # the areas, one behind the other
    tile_rows = 16 * p["mt"]
    stage = p["mt"] * (1024 + 128 // group * 32)
    at = p["warps"] * p["stages"] * stage
    assert at % 16 == 0
    red = at
    if not p["direct"]:
        at += p["warps"] * columns * (tile_rows + 4) * 4
    part = at
    part_tokens = -(-p["per_pass"] // p["split"]) if p["split"] > 1 else 0
    at += 2 * groups * p["split"] * part_tokens * tile_rows * 4
    starts = at
    at += p["chunk"] * (128 // group) * 8 * p["nt"] * 4
    xs = at
    stride = p["chunk"] * 256 + 64
    assert red % 4 == 0 and part % 4 == 0 and starts % 8 == 0 and xs % 16 == 0, case
    # the furthest that is touched of each: a column of sums, another CTA's sums, the start of a group, a piece of x
    if not p["direct"]:
        assert red + ((p["warps"] * columns - 1) * (tile_rows + 4) + tile_rows) * 4 <= part, case
    if p["split"] > 1:
        last = (((1 * groups + groups - 1) * p["split"] + p["split"] - 1) * part_tokens + (p["per_pass"] - 1) // p["split"]) * tile_rows + tile_rows
        assert part + last * 4 <= starts, case
    assert starts + ((p["chunk"] * (128 // group) - 1) * 8 * p["nt"] + 8 * (p["nt"] - 1) + 8) * 4 <= xs, case
    assert xs + (columns - 1) * stride + ((p["chunk"] - 1) * 16 + 15) * 16 + 16 <= p["smem"], case


def test_listed_shapes():
    rows = (1, 16, 17, 144, 1000, 2048, 4097, 28672, 50257, 1 << 20)
    cols = (1, 128, 129, 400, 2048, 5003, 8192, 25088, 65536, 1000003)
    tokens = (1, 2, 3, 7, 8, 9, 16, 17, 21, 22, 33, 64, 65, 1000)
    for r, c, g, k, t in itertools.product(rows, cols, (32, 128), (0, 1), tokens):
        check(r, c, g, k, t)


def test_random_shapes_and_devices():
    r = random.Random(1)
    for _ in range(20000):
        check(int(2 ** r.uniform(0, 20)), int(2 ** r.uniform(0, 20)), r.choice([32, 64, 128]), r.choice([0, 1, 2]), int(2 ** r.uniform(0, 8)), r.choice([148, 148, 132, 16, 1]))
