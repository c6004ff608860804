"""The chunk attention's notes on non-finite V entries (tcgen05 kernel), in slots that are used again.  The warp that writes them
may not reset a slot while a softmax warp still reads it.  A sub-tile without keys in a segment meets no barrier there, so a slot
that both sub-tiles read by the segment's number could be reset under the slower one; each has slots by its own segments.  Nothing
on a GPU can be made to show that: the indexes are read from the source, and a model of the roles runs through every
interleaving."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_03700_gb300", "csrc")


def kernel():
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, "attention_chunk_tc.cuh")).read(), flags=re.S)
    at = text.index("chunk_tc_kernel(")
    return text[at:text.index("__global__", at)]


def test_each_sub_tile_has_slots_by_its_own_segments():
    k = kernel()
    # the softmax warps count the segments in which they have key tiles, and read their own slots
    assert re.search(r"n_my = g\.nt\(sub\);\s*seg \+= n_my > 0;", k)
    assert re.search(r"if \(n_my > 0 && s_poisoned\[sub\]\[seg & 3\]\)", k) and "s_pk[sub][seg & 3][e] < lim" in k
    # the writer counts the same, marks a slot empty where the sub-tile has key tiles in the segment, and notes keys of those tiles only
    for t in "01":
        assert f"seg{t} += g.nt{t} > 0;" in k
        assert f"if (lane == 0 && g.nt{t} > 0) s_poisoned[{t}][seg{t} & 3] = 0;" in k
        assert f"of{t} = j < g.nt{t}" in k
        assert f"if (of{t}) note({t}, seg{t} & 3);" in k
        assert f"if (of{t}) atomicMin(&s_pk[{t}][seg{t} & 3][col + e], k0 + key);" in k
    # the first note of a segment empties the columns
    assert re.search(r"if \(s_poisoned\[sub\]\[slot\]\) return;\s*__syncwarp\(\);\s*for \([^)]*\) s_pk\[sub\]\[slot\]\[e\] = 0x7fffffff;"
                     r"\s*s_poisoned\[sub\]\[slot\] = 1;\s*__syncwarp\(\);", k)
    # nothing else names them
    assert len(re.findall(r"\bs_(?:pk|poisoned)\b", k)) == 2 + 2 + 2 + 2 + 3


def every_order(has, slots_per_sub):
    """Whether some interleaving lets a sub-tile find its slot reset for a later segment.  has[sub][s]: the sub-tile has key tiles in
    segment s (of one key tile, the tightest).  Steps: the writer resets the slots of its next segment w, once V of segment w - 2 is
    through, which takes a P of each sub-tile that has keys there; a sub-tile hands over P of its next segment, then reads its
    notes."""
    n = len(has[0])
    own = [[s for s in range(n) if h[s]] for h in has]

    def slot(sub, s):
        return (own[sub].index(s) if slots_per_sub else s) % 4

    bad, ends, seen, todo = False, False, set(), [(0, (0, 0))]   # segments written; steps taken (two a segment) per sub-tile
    while todo:
        at = todo.pop()
        if at in seen:
            continue
        seen.add(at)
        w, steps = at
        ends |= w == n and all(steps[i] == 2 * len(own[i]) for i in (0, 1))
        through = w < 2 or all(not has[i][w - 2] or steps[i] > 2 * own[i].index(w - 2) for i in (0, 1))
        if w < n and through:
            todo.append((w + 1, steps))
        for i in (0, 1):
            k, reading = divmod(steps[i], 2)
            if k == len(own[i]) or own[i][k] >= w:
                continue
            if reading:
                s = own[i][k]
                later = [x for x in range(s + 1, w) if (has[i][x] if slots_per_sub else True) and (slot(i, x) if slots_per_sub else x % 4) == slot(i, s)]
                bad |= bool(later)
            todo.append((w, tuple(steps[j] + (j == i) for j in (0, 1))))
    assert ends, "stuck"
    return bad


PATTERNS = [
    ((1, 1, 1, 1, 1, 1, 1), (1, 0, 0, 0, 0, 0, 1)),
    ((1, 1, 1, 1, 1, 1, 1, 1), (0, 1, 0, 0, 0, 1, 0, 0)),
    ((1, 0, 0, 0, 0, 0, 1), (0, 1, 1, 1, 1, 1, 1)),
    ((1, 0, 1, 1, 1, 0, 1), (1, 1, 0, 0, 1, 1, 1)),
    ((1,) * 9, (1,) * 9),
    ((0, 1, 1, 0, 0, 1, 1, 0, 1, 1), (1, 0, 0, 1, 1, 1, 0, 1, 1, 0)),
]


@pytest.mark.parametrize("has", PATTERNS, ids=str)
def test_slots_by_a_sub_tiles_own_segments_hold(has):
    assert not every_order(has, slots_per_sub=True)


@pytest.mark.parametrize("has", PATTERNS[:3], ids=str)
def test_slots_by_the_segments_number_would_not(has):
    assert every_order(has, slots_per_sub=False)
