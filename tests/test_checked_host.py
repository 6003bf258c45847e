"""Indices that data decide go through the check of the range-checked build, in the kernels on tokens as elsewhere: without it that build's count of faults says nothing of them."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_26845_b200", "csrc")

# what a chosen expert, a place in a warp's list, or a slot may stand in, and at least how often
PLACES = {
    "choose_kernel.cu": (r"\b(?:own|bias)\[(expert)\b", r"\blist\[(at\+\+)", r"\blist\[(?:32 \+ )?(place)\b", r"\bout \+ (expert)\b", 8),
    "rows_kernel.cu": (r"\bfirst \+ (to)\b", r"\bfirst\([^()]*\) \+ (from)\b", r"\* rows \+ (at)\b", 4),
}


@pytest.mark.parametrize("name", PLACES)
def test_places_that_data_decide_are_checked(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//.*", "", f.read())
    *patterns, least = PLACES[name]
    for pattern in patterns:
        assert not re.search(pattern, text), pattern
        checked = pattern.replace("(expert)", r"MS_AT\(expert").replace(r"(at\+\+)", r"MS_AT\(at\+\+").replace("(place)", r"MS_AT\(place")
        checked = checked.replace("(to)", r"MS_AT\(\(int\)to").replace("(from)", r"MS_AT\(\(int\)from").replace("(at)", r"MS_AT\(at")
        assert re.search(checked, text), checked
    assert len(re.findall(r"\bMS_AT\(", text)) >= least
