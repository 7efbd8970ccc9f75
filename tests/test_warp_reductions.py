"""Warp-wide calls with a full mask, checked on the sources (no GPU): every lane has to make the call at the same place.  One in an
arm of a conditional expression is made at two places, by the lanes of either condition apart, unless the compiler
happens to merge them."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_15618_b200", "csrc")
FILES = ("fm_logprobs.cuh", "fm_pages.cuh", "fm_tree.cuh", "fm_hourglass_tree.cuh")
CALL = re.compile(r"__(?:reduce_\w+|shfl\w*|ballot|any|all|match_\w+)_sync\(0xffffffffu|warp_(?:max|sum|sort)\(|__syncwarp\(")


def _statements(text):
    text = re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))
    return [s.strip() for s in re.split(r"[;{}]", text)]


def _arms(statement):
    """What stands behind the first question mark of a conditional expression, outside of brackets that enclose it."""
    at = statement.find("?")
    return statement[at + 1:] if at >= 0 else ""


def test_no_full_mask_call_in_an_arm_of_a_condition():
    seen, bad = 0, []
    for f in FILES:
        for s in _statements(open(os.path.join(CSRC, f)).read()):
            seen += bool(CALL.search(s))
            if CALL.search(_arms(s)):
                bad.append((f, " ".join(s.split())))
    assert seen > 40
    # (a condition that is the same for the whole warp: the constant of an instance, an argument of the launch)
    assert not bad, bad
