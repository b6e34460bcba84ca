"""Orderings of tensor-memory accesses that no run can show to be missing, read from the kernels' sources (CPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21862_b200", "csrc")


def lambda_body(source, name):
    """Text between the braces of `auto name = [...](...) { ... }`, comments taken out."""
    source = re.sub(r"//[^\n]*", "", source)
    start = source.index("{", source.index(f"auto {name} = [&]("))
    depth = 0
    for i in range(start, len(source)):
        depth += {"{": 1, "}": -1}.get(source[i], 0)
        if depth == 0:
            return source[start + 1: i]
    raise AssertionError(name)


def test_pipelines_read_each_others_accumulators_behind_a_fence():
    """tree_tok_kernel merges its two pipelines at a unit's end: every softmax warp reads both accumulators, but has itself
    waited only for its own pipeline's MMAs.  The barrier in between orders the reads only with a fence on either side."""
    with open(os.path.join(CSRC, "tree_kernels.cuh")) as f:
        source = f.read()
    meet = lambda_body(source, "both_sync")
    before, arrive, wait, after = (meet.find(s) for s in ("tc_fence_before_sync()", "mbar_arrive(s_both)", "tok_wait(s_both",
                                                          "tc_fence_after_sync()"))
    assert 0 <= before < arrive < wait < after, (before, arrive, wait, after)
    finish = lambda_body(source, "finish_unit")
    assert 0 <= finish.index("both_sync()") < finish.index("tmem_ld16(")
