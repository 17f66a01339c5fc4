"""Memory order in draft verification's kernels, by reading (CPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_00835_gb300", "csrc")


def test_all_lanes_read_shares_behind_the_fence():
    """A row's last share is counted by one lane, between two fences; the others read what other CTAs wrote only
    behind a barrier of the warp, which orders memory where a shuffle need not."""
    with open(os.path.join(CSRC, "verify.cu")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    reads = [m.start() for m in re.finditer(r"__ldcg\(a\.shares", code)]
    assert len(reads) == 1
    before = code[code.rindex("atomicAdd(&a.row_tickets", 0, reads[0]):reads[0]]
    steps = [before.find(s) for s in ("__threadfence();", "__shfl_sync(~0u, last, 0)", "__syncwarp();")]
    assert -1 not in steps and steps == sorted(steps)
