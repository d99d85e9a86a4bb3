"""The hand-overs between the two CTAs of a pair in the 4-bit products, read from the source: an order of memory that is missing there shows in no run."""
import os
import re

import paper_2607_18002_b200 as moe

SOURCE = os.path.join(os.path.dirname(moe.__file__), "csrc", "moe_mx_product.cu")


def _code():
    with open(SOURCE) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_what_one_cta_hands_to_the_other_is_ordered_for_the_cluster():
    """An arrival on the other CTA's barrier by a thread that wrote or read shared memory or TMEM releases to the cluster, and the wait behind it acquires from
    there: by their own semantics, or by a fence directly before the one and one behind the other."""
    code = re.sub(r"\s+", " ", _code())
    arrivals = re.findall(r"(\w+\(\); )?(\w+)\(map_to_cta\(&s\.(\w+)", code)
    assert {bar for _, _, bar in arrivals} == {"landed", "acc_empty"}
    for before, call, bar in arrivals:
        fenced = call == "mbar_arrive_relaxed"
        assert before == "fence_release_own_smem(); " if fenced else call == "mbar_arrive_cluster", (call, bar)
        waits = re.findall(r"wait(<[^(]*>)?\(&s\.%s\[[^;]*;( if \(!ok\) break; if \(kPair\) fence_acquire_pair_smem\(\);)?" % bar, code)
        assert len(waits) == 1, (bar, waits)
        kind, behind = waits[0]
        assert kind == "<kPair ? %s : mbar_try>" % ("mbar_try_relaxed" if fenced else "mbar_try_cluster") and bool(behind) == fenced, (bar, waits)


def test_copies_in_flight_are_waited_for_whatever_ended_the_launch():
    """Shared memory is not given back under a copy: the thread that issued the copies looks at all that may be outstanding when it is done, also where another
    role gave up after it, and within one limit for all of them."""
    code = re.sub(r"\s+", " ", _code())
    at = code.index("tma_2d<kPair>(to + S::kWBytes")
    tail = code[at:code.index("__syncwarp()", at)]
    limit, loop = tail.index("start = gtime_ns()"), tail.index("for (unsigned m")
    head = tail[loop:tail.index(")", tail.index("++m"))]
    assert "dead" not in head and "n > S::kStages ? n - S::kStages : 0" in head and "m < n" in head
    assert limit < loop and tail.count("gtime_ns()") == 2 and "gtime_ns() - start < kWaitNs" in tail[loop:]
