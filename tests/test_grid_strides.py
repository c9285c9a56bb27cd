"""Loops that a grid shares out: their counters hold any number of threads that a launch can have.  Host only."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_20390_amd", "csrc")


def test_counters_of_shared_loops_have_64_bits():
    """The step of such a loop is the grid's number of threads, up to 2^32: a counter of 32 bits that is added to it comes out below zero, which is below
    any limit."""
    loops = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        for line in open(path):
            m = re.search(r"for \((.*?) (\w+) = .*blockIdx.*;.*\2 \+= .*gridDim", line)
            if m:
                loops.append((os.path.basename(path), m.group(1)))
    assert loops and all(kind == "int64_t" for _, kind in loops), loops
