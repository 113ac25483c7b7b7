"""Waits of the kernels, as the sources have them: mbar_wait_bounded answers for one lane, so where a whole warp waits and goes on to instructions that
need all its lanes (tcgen05.ld, elect.sync, barriers of the warp) the answer has to be the warp's, or lanes that disagree when the limit runs out
leave the others waiting for them without a limit."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_12801_b200", "csrc")
ONE_LANE = re.compile(r"lane == 0|threadIdx\.x ==|struct NormFeed")      # NormFeed is used by lane 0 of the producer's warp
# the norms' consumers go on through their shuffles and barriers whatever the answer, and vote on it at the end
VOTED_LATER = re.compile(r"struct NormGroup")
CALL = re.compile(r"\bmbar_wait_(bounded|cluster)\(")


def waits(text):
    """(line number, whether the call is guarded) for each call: guarded by an enclosing block, by its own statement or by a vote around it."""
    text = re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), text)
    calls, stack, start = [m.start() for m in CALL.finditer(text)], [], 0
    for i, ch in enumerate(text):
        if i in calls:
            head = text[start:i]
            if "__device__" not in head:                                  # not the definition
                around = stack + [head]
                yield text.count("\n", 0, i) + 1, any(ONE_LANE.search(h) or VOTED_LATER.search(h) for h in around) or "__all_sync(" in head
        if ch == "{":
            stack.append(text[start:i])
        elif ch == "}" and stack:
            stack.pop()
        if ch in "{};":
            start = i + 1


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_waits_of_a_warp_have_one_answer(path):
    if path.endswith("common.cuh"):
        pytest.skip("the wait itself")
    open_ones = [line for line, guarded in waits(open(path).read()) if not guarded]
    assert open_ones == [], f"{os.path.basename(path)}: lanes of a warp may disagree at lines {open_ones}"


def test_the_warps_wait_votes():
    text = open(os.path.join(CSRC, "common.cuh")).read()
    body = text[text.index("bool mbar_wait_warp("):]
    body = body[:body.index("\n}")]
    assert "if (__all_sync(0xffffffffu, mbar_try_wait(bar, phase))) return true;" in body and "it < limit" in body


def test_the_norms_vote_at_the_end():
    text = open(os.path.join(CSRC, "norm.cuh")).read()
    assert "norm_ring_end(group.ok" not in text and text.count("norm_ring_end(__all_sync(0xffffffffu, group.ok), error_flag);") == 2


def test_the_check_sees_what_it_is_for():
    assert [ok for _, ok in waits("void f() { if (lane == 0) { ok = mbar_wait_bounded(&b, 0); } ok = mbar_wait_bounded(&b, 1); }")] == [True, False]
    assert [ok for _, ok in waits("x = __all_sync(0xffffffffu, mbar_wait_cluster(&b, 0)); y = mbar_wait_cluster(&b, 0);")] == [True, False]
