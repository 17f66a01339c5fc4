"""The paged cache's kernels may start while the kernel before them in the stream is still
writing what they will read (lengths, tables, slots, masks, the rotary table): they
wait, and then read it with coherent loads only."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_00835_gb300", "csrc")


def test_no_non_coherent_load():
    files = glob.glob(os.path.join(CSRC, "paged*.cu*"))
    assert len(files) >= 8
    for f in files:
        with open(f) as fh:
            code = re.sub(r"//[^\n]*", "", fh.read())
        assert not re.search(r"__ldg\b|__restrict|ld\.global\.(\w+\.)*nc\b", code), os.path.basename(f)


def test_kernels_wait_before_they_read():
    """Every kernel of these files has its wait, and starts by a launch that allows the overlap."""
    kernels = 0
    for f in glob.glob(os.path.join(CSRC, "paged*.cu")):
        with open(f) as fh:
            code = fh.read()
        n = len(re.findall(r"__global__", code))
        assert code.count("pdl_wait();") >= n, os.path.basename(f)
        kernels += n
    assert kernels >= 5
