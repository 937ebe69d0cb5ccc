"""What the warps of attention's tile kernel read of each other, and behind which waits: looked up in its source. CPU only."""
import re

import pytest

from test_memory_order import body


@pytest.fixture(scope="module")
def parts():
    """The kernel's text by the tasks of its warps."""
    text = body("lc_attend_tiles.cu", "void run(const AttendArgs& A)")
    cuts = ["if (warp < kSoftmaxWarps) {", "else if (warp < kSoftmaxWarps + 2 * kReadWarps) {", "if (warp < kSoftmaxWarps + 2 * kReadWarps + 2) {", "const uint32_t set = warp - (kSoftmaxWarps + 2 * kReadWarps + 2)"]
    at = [text.index(c) for c in cuts] + [len(text)]
    assert at == sorted(at)
    return dict(zip(("scores", "readers", "issue", "lookup"), (text[a:b] for a, b in zip(at, at[1:]))))


def test_a_tiles_units_are_read_behind_the_wait_for_its_values(parts):
    # The warps that look up values write them ahead of found_full, which the readers of values wait for ahead of full_v. A block's first scores depend on its
    # keys alone, so the warps of the scores wait for full_v themselves.
    text = parts["scores"]
    loop = text.index("; i < 2 * n; ++i) {")
    scores, read = text.index("warp_wait(shared_address(&S.scores[t][half])", loop), text.index("S.value_units[", loop)
    wait = re.search(r"if \(i == 0 && !warp_wait\(shared_address\(&S\.full_v\[2 \* done % kStages\]\), 2 \* done / kStages & 1, dead\)\) break;", text[scores:read])
    assert wait
    assert "S.value_units[" not in text[:scores]  # nor ahead of the loop
    # a half's place among the operands: one counter over all halves of all blocks
    assert "if (++stage == kStages) stage = 0, ++turn;" in parts["readers"] and "if (++v_stage == kStages) v_stage = 0, ++v_turn;" in parts["issue"]


def test_later_tiles_units_are_written_ahead_of_their_scores(parts):
    # half i + 2 of the scores is issued behind half i of the values, and that is stored once the tile of half i + 2 has been looked up
    issue = parts["issue"]
    loop = issue.index("for (uint32_t i = 0; i < 2 * n && good; ++i) {")
    assert 0 < issue.index("S.full_v[v_stage]", loop) < issue.index("multiply_keys(half, k_stage)", loop)
    assert "const bool more = i + 2 < 2 * n;" in issue
    readers = parts["readers"]
    loop = readers.index("for (uint32_t i = 0; i < 2 * n; ++i) {")
    assert 0 < readers.index("if (n > 1) {") < readers.index("good = found(1);") < loop
    assert 0 < readers.index("store_numbers(", loop) < readers.index("if (i & 1) good = found((i + kAhead) / 2);", loop)
    text = body("lc_attend_tiles.cu", "namespace lc {")
    assert int(re.search(r"constexpr uint32_t kAhead = (\d+);", text).group(1)) == 3  # found((i + 3) / 2) at odd i is the tile behind half i's
    lookup = parts["lookup"]
    assert lookup.index("S.value_units[") < lookup.index("barrier_arrive(shared_address(&S.found_full[set][slot]))")


def test_the_warps_of_the_scores_look_nothing_up(parts):
    # Which queries see values that are no numbers is noted by the warp that looks those up. (A walk through a block's keys by every thread of the scores, behind one
    # such value, can take longer than the other warps wait for.) The notes are read once the sums are there, and no way that a warp takes as a whole hangs on them.
    text = parts["scores"]
    assert not re.search(r"\b(page_of|place_of_key)\(|A\.scales|A\.table", text)
    read = [m.start() for m in re.finditer(r"S\.broken", text)]
    assert len(read) == 1 and read[0] > text.index("warp_wait(shared_address(&S.sums[t][h]), (done + n - 1) & 1, dead)")
    assert not re.search(r"if \([^)]*S\.broken", text)
    lookup = parts["lookup"]
    assert lookup.index("note_broken(") < lookup.index("barrier_arrive(shared_address(&S.found_full[set][slot]))")
