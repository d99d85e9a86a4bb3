"""What a product of e4m3 rows leaves when a wait inside its kernel runs out: rows that are right, or that say that they are not."""
import os
import re

import paper_2607_18002_b200 as moe

SOURCE = os.path.join(os.path.dirname(moe.__file__), "csrc", "moe_scaled_product.cu")


def _code():
    with open(SOURCE) as f:
        return re.sub(r"\s+", " ", re.sub(r"//[^\n]*", "", f.read()))


def test_nothing_is_given_back_that_was_waited_for_in_vain():
    """A warp that gave up does not arrive on the barriers that let partials and scales be overwritten: the other warps may not have read them yet.  Every hand-over behind a
    wait in the same step asks for its answer."""
    code = _code()
    epilogue = code[code.index("const auto next_partial"):code.index("if (warp == kTmaWarp)")]
    waits = list(re.finditer(r"(next_partial|next_scales)\(\)", epilogue))
    gives = list(re.finditer(r"(if \(ok\) )?(hand_back|scales_read)\(\);", epilogue))
    assert len(gives) == 8
    for g in gives:
        wait = "next_partial" if g[2] == "hand_back" else "next_scales"
        before = max(w.end() for w in waits if w[1] == wait and w.end() < g.start())
        between = epilogue[before:g.start()]
        # ... directly, or by a loop that begins with it, or by the loads in between that are left out
        assert g[1] or "if (!ok) break;" in between or re.search(r"&& ok; (\+\+b|b0 \+= 2)\)", between), epilogue[before - 40:g.end()]
