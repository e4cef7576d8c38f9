"""Faults of the attention operators that reading or the CPU can show: what a kernel's wavefronts hand to each other, what its loads
reach, what the entry points refuse.  No GPU needed."""
import os
import re

from paper_2407_00088_amd import build


def source(name):
    return open(os.path.join(build.CSRC, name)).read()


def body_of(src, head):
    """The text between the braces that open after `head`."""
    at = src.index("{", src.index(head))
    depth = 0
    for i in range(at, len(src)):
        depth += {"{": 1, "}": -1}.get(src[i], 0)
        if depth == 0:
            return src[at:i + 1]
    raise AssertionError(head)


def test_sums_of_rows_are_handed_over_before_the_last_barrier():
    """The decode kernel of whole rows reads row_lse in every wavefront right after `finish`, whose first wavefront writes it."""
    src = source("tmac_attn.hip")
    finish = body_of(src, "void finish(")
    writes = [m.start() for m in re.finditer(r"row_lse\[", finish)]
    assert writes and max(writes) < finish.rindex("__syncthreads()")
