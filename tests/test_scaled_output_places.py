"""Outputs of e4m3 products on their way out of shared memory: a warp's places and the waits before they are written again, read from the source."""
import os
import re

import pytest

import paper_2607_18002_b200 as moe

SOURCE = os.path.join(os.path.dirname(moe.__file__), "csrc", "moe_scaled_product.cu")


def _waits(turns):
    """pass of a tile -> how many of the warp's latest stores may be left unread, or None: no wait; as the code says."""
    with open(SOURCE) as f:
        code = re.sub(r"\s+", " ", re.sub(r"//[^\n]*", "", f.read()))
    guard, first, left = re.search(r"if \(kForm != kNarrow( && [^{]*)?\) \{ if \(lane == 0\) \{ if \(([^)]*)\) tma_stores_read<0>\(\); else tma_stores_read<([^>]*)>\(\);", code).groups()
    names = dict(turns=turns)
    py = lambda text: text.replace("S::kTurns", "turns").replace("&&", "and").replace("||", "or")
    return lambda c: None if guard and not eval(py(guard).strip().removeprefix("and "), dict(names, c=c)) else 0 if eval(py(first), dict(names, c=c)) else eval(py(left), names)


@pytest.mark.parametrize("turns", [1, 2, 4])
@pytest.mark.parametrize("passes", [1, 2, 4])
def test_a_place_is_free_when_it_is_written_and_nothing_else_is_waited_for(turns, passes):
    waits, stored, read = _waits(turns), [], 0        # places of the stores so far, and how many of the oldest are known to be read
    for tile in range(3):
        for c in range(passes):
            left = waits(c)
            if left is not None:
                done = max(read, len(stored) - left)
                # within a tile, no store is waited for but the one whose place comes again (between tiles all of them are)
                assert c == 0 or all(p == c % turns for p in stored[read:done]), (tile, c)
                read = done
            assert c % turns not in stored[read:], (tile, c)
            stored.append(c % turns)
