"""Waits on barriers that threads of the peer CTA arrive on, by the kernels' source (no GPU).

A thread of the other CTA of a pair releases at cluster scope. Only an acquire at cluster scope orders what follows
a wait behind what that thread did; the plain waits acquire within their own CTA. A missing one shows in no run
that can be relied on, so it is looked for in the text."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_04526_gb300", "csrc")
WAIT = re.compile(r"\b(\w*(?:wait|spin|test)\w*)(<\w+>)?\(&?(\w+)(?:\[[^\]]*\])?")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def waits(text, barrier):
    """(function, template argument) of every wait on a barrier in kernel code."""
    return [(m[1], m[2] or "") for m in WAIT.finditer(text) if m[3] == barrier]


def at_cluster_scope(function, argument):
    return "cluster" in function or argument == "<true>"


@pytest.mark.parametrize("name, barriers", [("sq_gemm_kernels.cuh", ("tempty", "pready")), ("sq_loss.cu", ("tempty",)),
                                            ("sq_fp4.cu", ("tempty",))])
def test_barriers_of_both_ctas_are_acquired_at_cluster_scope(name, barriers):
    text = source(name)
    for barrier in barriers:
        found = waits(text, barrier)
        assert found, f"no wait on {barrier} in {name}"
        assert all(at_cluster_scope(*w) for w in found), f"{name}: {barrier} is waited for by {found}"


def test_stages_that_the_peer_mends_are_acquired_at_cluster_scope():
    """The 4-bit pair kernel: the leader's MMAs of a stage whose codes both CTAs have changed."""
    text = source("sq_fp4.cu")
    issue = text[text.index("MMA issuer (leader"):text.index("codes of blocks with a negative scale", text.index("MMA issuer (leader"))]
    found = waits(issue, "full")
    assert len(found) == 3 and all(w[1] == "<kMended>" for w in found), found
    mended = re.search(r"__any_sync\(0xFFFFFFFFu, mend\)\)\s*issue\(std::true_type\(\)\);\s*else\s*issue\(std::false_type\(\)\);", issue)
    assert mended, "the loop over mended stages is chosen by what the launch met"
    assert re.search(r"return CLUSTER \? mbar_test_wait_cluster\(bar, parity\) : mbar_test_wait\(bar, parity\);", text)
