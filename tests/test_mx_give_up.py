"""What a 4-bit product's warps give back after a wait that ran out, read from the source."""
import os
import re

import paper_2607_18002_b200 as moe

SOURCE = os.path.join(os.path.dirname(moe.__file__), "csrc", "moe_mx_product.cu")


def test_an_accumulator_that_was_waited_for_in_vain_is_not_given_back():
    """The other warps may still read the one before it in the same place; the barrier that lets it be overwritten counts all of them."""
    with open(SOURCE) as f:
        code = re.sub(r"\s+", " ", re.sub(r"//[^\n]*", "", f.read()))
    arrivals = [m.start() for m in re.finditer(r"mbar_arrive\w*\((map_to_cta\()?&s\.acc_empty", code)]
    assert len(arrivals) == 2
    for at in arrivals:
        assert "if (lane == 0 && ok)" in code[code.rindex("__syncwarp()", 0, at):at]
