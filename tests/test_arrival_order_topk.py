"""The top-log-probability loss is summed by the cluster that finds itself the last: the count goes through the helper that
fences on both sides, one thread counts, and barriers stand before it and between it and the sums (no run can be made to
fail without them, so the order is read off the source)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_27233_gb300", "csrc")


def test_the_last_cluster_is_counted_between_barriers():
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "distill_topk.cu")).read())
    assert code.count("arrive_is_last(") == 1
    assert re.search(r"__syncthreads\(\);\s*if \(tid == 0\) \{\s*s_last = 0;\s*if \(arrive_is_last\([^;]*\)\) s_last = 1;\s*\}"
                     r"\s*__syncthreads\(\);\s*if \(!s_last\) return;", code)
    assert "__ldcg(a.pair_loss" in code[code.index("arrive_is_last("):]   # the others' losses, not this SM's cache
